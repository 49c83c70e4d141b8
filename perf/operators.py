"""The operators around the window selection, as timed cases: what an engine runs before it (rotary positions, the
prompt's attention with the normalisers that the selection takes) and after it (new tokens appended to the paged compact
cache and attending over it, rows leaving the cache by their accumulated attention weight).

Where `own` is false, `run` computes them from elementary tensor operations; where it is true, it calls the entry points of
`paper_2503_17922_b200.binding`.

Fields of a case:
  op         "prompt"   causal attention of whole prompts, with the log-sum-exp of every row and of the observation rows
             "attend"   attention of new tokens over a paged cache, optionally adding up the weight that each row receives
             "rotate"   rotary positions of a prompt's queries and keys
             "append"   rotary positions of new tokens, their keys and values written into the paged cache
             "evict"    the rows of least accumulated weight leave the cache, in place, for every layer of a group
  dtype      "bf16" or "f32";  batch, q_heads, kv_heads, d: attention shape
  n          prompt length (prompt, rotate) or rows in the cache, new ones included (attend, append, evict): the longest
  ragged     lengths between n / 2 and n; prompts and chunks of new tokens are packed [T, heads, d]
  layout     "bhnd" or "bnhd" (token-major) for dense prompts, "phsd" or "pshd" (token-major) for pages
  new        new tokens of a sequence (the most, when ragged);  page: rows of a page
  weights    attend: with accumulated weights
  rot        rotated dimensions;  order: "half" or "interleaved";  scaling: "none", "linear", "base" or "bands"
  at         append: position of a sequence's first new token
  layers     evict: layers that share the selection;  budget: rows kept;  recent: newest positions that always stay
"""
import math

import torch

own = False

_LARGEST = {"bytes": 2.0e9, "flops": 8.9e12}     # what the largest listed cases cannot do without
_BASE = 500000.0
_FACTOR, _ORIGINAL, _LOW, _HIGH = 8.0, 8192, 1.0, 4.0     # scaling for long contexts


def _case(op, **kw):
    c = dict(op=op, dtype="bf16", batch=1, q_heads=32, kv_heads=8, d=128, ragged=False)
    c.update(kw)
    return c


def listed():
    return [
        # a unit test's or a toy model's prompt in fp32: nothing but latency
        _case("prompt", name="tiny-prompt-f32", dtype="f32", q_heads=4, kv_heads=2, d=64, n=1024, alpha=8, layout="bhnd"),
        # an ordinary prompt of one layer
        _case("prompt", name="8k-prompt", n=8192, alpha=32, layout="bhnd"),
        # a packed batch of prompts of odd lengths, six query heads per key head
        _case("prompt", name="g6-ragged-prompts", batch=3, q_heads=12, kv_heads=2, n=12289, alpha=16, ragged=True, layout="bnhd"),
        # full context, token-major tensors: the largest
        _case("prompt", name="32k-prompt", n=32768, alpha=32, layout="bnhd"),
        # one sequence's next token over the 12 percent of an 8 K prompt that were kept: latency
        _case("attend", name="one-token", n=992, new=1, page=16, layout="phsd", weights=False),
        # a decoding batch over long caches of different lengths, whose rows' weights are added up for the eviction
        _case("attend", name="token-batch", batch=32, n=8192, new=1, page=64, layout="pshd", ragged=True, weights=True),
        # chunks of a batch's next prompt parts over what is cached already
        _case("attend", name="chunk-16k", batch=4, n=16384, new=512, page=128, layout="phsd", ragged=True, weights=False),
        # fp32, pages of an odd number of rows, a few tokens at once
        _case("attend", name="tiny-attend-f32", dtype="f32", batch=3, q_heads=4, kv_heads=2, d=64, n=1027, new=7, page=24,
              layout="phsd", ragged=True, weights=True),
        # the same decoding batch's step before its attention: far positions under a scaled context
        _case("append", name="append-batch", batch=32, n=8192, new=1, page=64, layout="pshd", ragged=True, rot=128, order="half",
              scaling="bands", at=100000),
        # a whole prompt's queries and keys, half of each head rotated
        _case("rotate", name="rotate-32k", n=32768, layout="bnhd", rot=64, order="interleaved", scaling="linear"),
        # one sequence's cache back to its budget, four layers that share their rows
        _case("evict", name="evict-one", n=992, page=16, layout="phsd", layers=4, budget=983, recent=32),
        # a batch of long caches to half their rows
        _case("evict", name="evict-batch", batch=16, n=8192, page=64, layout="pshd", ragged=True, layers=4, budget=3932, recent=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))


def draw(rng):
    while True:
        op = rng.choice(["prompt", "attend", "attend", "append", "rotate", "evict"])
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        c = _case(op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), batch=_log_int(rng, 1, 32),
                  q_heads=kv_heads * rng.choice([1, 2, 3, 4, 6, 8]), kv_heads=kv_heads, d=rng.choice([64, 80, 96, 128]),
                  ragged=rng.random() < 0.5)
        if op in ("prompt", "rotate"):
            c.update(n=_log_int(rng, 1, 16384), layout="bnhd" if c["ragged"] else rng.choice(["bhnd", "bnhd"]))
        else:
            c.update(n=_log_int(rng, 1, 16384), page=rng.choice([8, 16, 24, 32, 64, 128]), layout=rng.choice(["phsd", "pshd"]))
        if op == "prompt":
            c.update(alpha=rng.choice([1, 8, 16, 32, 64]))
        if op in ("attend", "append"):
            c.update(new=min(c["n"], 1 if rng.random() < 0.4 else _log_int(rng, 1, 512)))
        if op == "attend":
            c.update(weights=rng.random() < 0.5)
        if op in ("append", "rotate"):
            c.update(rot=2 * rng.randint(1, c["d"] // 2), order=rng.choice(["half", "interleaved"]),
                     scaling=rng.choice(["none", "linear", "base", "bands"]))
        if op == "append":
            c.update(at=_log_int(rng, 1, 1000000))
        if op == "evict":
            c.update(layers=rng.randint(1, 8), budget=rng.randint(0, c["n"]), recent=_log_int(rng, 1, 512) - 1)
        w = work(c)
        f32_limit = 0.02 if c["dtype"] == "f32" else 0.25
        if w["bytes"] <= _LARGEST["bytes"] and w["flops"] <= f32_limit * _LARGEST["flops"] and _scores(c) <= 2 ** 32 and _cache_bytes(c) <= 4e9:
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


def _scores(c):
    """Scores that the plain form of an "attend" case holds at once."""
    return c["batch"] * c["q_heads"] * c["new"] * c["n"] if c["op"] == "attend" else 0


def _cache_bytes(c):
    if c["op"] in ("prompt", "rotate"):
        return 0
    return 2.0 * c.get("layers", 1) * c["batch"] * (c["n"] + c["page"]) * c["kv_heads"] * c["d"] * _elem(c)


def work(case):
    c = case
    e, d, hq, hk = _elem(c), c["d"], c["q_heads"], c["kv_heads"]
    lens = _lengths(c)
    if c["op"] == "prompt":
        pairs = sum(n * (n + 1) / 2 for n in lens)
        rows = sum(lens)
        lse = 4.0 * hq * (rows + sum(min(n, c["alpha"]) for n in lens))
        return {"bytes": rows * (2.0 * hq + 2.0 * hk) * d * e + lse, "flops": 4.0 * d * hq * pairs}
    if c["op"] == "rotate":
        return {"bytes": 2.0 * sum(lens) * (hq + hk) * d * e, "flops": 3.0 * sum(lens) * (hq + hk) * c["rot"]}
    if c["op"] == "evict":
        # of the len - keep rows that leave, those in front of row `keep` (a share of keep / len of them) are filled from behind it
        moved = sum((n - min(n, c["budget"])) * min(n, c["budget"]) / n for n in lens)
        state = sum(8.0 * n + 8.0 * min(n, c["budget"]) for n in lens)
        return {"bytes": hk * (moved * c["layers"] * 4.0 * d * e + state), "flops": 0.0}
    news = _news(c)
    q = sum(news) * hq * d * e
    if c["op"] == "append":
        return {"bytes": 2.0 * q + 4.0 * sum(news) * hk * d * e, "flops": 3.0 * sum(news) * (hq + hk) * c["rot"]}
    pairs = sum(m * n - m * (m - 1) / 2 for m, n in zip(news, lens))
    state = 8.0 * hk * sum(lens) if c["weights"] else 0.0
    return {"bytes": 2.0 * q + 2.0 * sum(lens) * hk * d * e + state, "flops": 4.0 * d * hq * pairs}


# ---- what a program has in hand before the call ----------------------------------------------------
def _frequencies(c):
    """Angle per position of every rotated pair (on the host, 64 bits)."""
    rot = c["rot"]
    i = torch.arange(rot // 2, dtype=torch.float64)
    base = _BASE
    if c["scaling"] == "base" and rot > 2:
        base *= _FACTOR ** (rot / (rot - 2))
    f = base ** (-2.0 * i / rot)
    if c["scaling"] == "linear":
        f = f / _FACTOR
    if c["scaling"] == "bands":
        turns = _ORIGINAL * f / (2.0 * math.pi)      # of a pair over the original context
        keep = ((turns - _LOW) / (_HIGH - _LOW)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / _FACTOR)
    return f


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dtype(c)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    B, hq, hk, d = c["batch"], c["q_heads"], c["kv_heads"], c["d"]
    s = {"case": c, "lens": _lengths(c)}
    if c["op"] in ("prompt", "rotate"):
        n, T = c["n"], sum(s["lens"])
        s["cu"] = _cu(s["lens"]) if c["ragged"] else None

        def heads(h):
            if c["ragged"]:
                return normal(T, h, d)
            return normal(B, h, n, d) if c["layout"] == "bhnd" else normal(B, n, h, d).transpose(1, 2)

        s["q"], s["k"] = heads(hq), heads(hk)
        s["q_out"] = torch.empty_like(s["q"])
        if c["op"] == "prompt":
            s["v"] = heads(hk)
            s["lse"] = torch.zeros((B, hq, n), device="cuda")
            s["lse_obs"] = torch.zeros((B, hq, c["alpha"]), device="cuda")
        else:
            s["k_out"] = torch.empty_like(s["k"])
            s["freq"] = _frequencies(c)
    else:
        page, n = c["page"], c["n"]
        max_pages = (n + page - 1) // page + 1
        num_pages = B * max_pages + 3
        s["max_pages"], s["num_pages"], s["capacity"] = max_pages, num_pages, max_pages * page
        order = torch.randperm(num_pages, generator=g, device="cuda")[: B * max_pages]
        s["table"] = order.view(B, max_pages).to(torch.int32)
        pool = (num_pages, hk, page, d) if c["layout"] == "phsd" else (num_pages, page, hk, d)
        s["k_pools"] = [normal(*pool) for _ in range(c.get("layers", 1))]
        s["v_pools"] = [normal(*pool) for _ in range(c.get("layers", 1))]
        # a head whose selection held the prompt's short last window has a few rows fewer
        rows = torch.tensor(s["lens"], device="cuda").view(B, 1) - torch.arange(hk, device="cuda").view(1, hk) % 3
        if c["op"] in ("attend", "append"):
            s["news"] = _news(c)
            news = torch.tensor(s["news"], device="cuda").view(B, 1)
            rows = torch.maximum(rows, news)
            s["cu"] = _cu(s["news"]) if c["ragged"] else None
            T = sum(s["news"])

            def chunk(h):
                return normal(T, h, d) if c["ragged"] else normal(B, h, c["new"], d)

            s["q"] = chunk(hq)
            s["q_out"] = torch.empty_like(s["q"])
        if c["op"] == "append":
            rows = rows - news
            s["k"], s["v"] = chunk(hk), chunk(hk)
            first = torch.repeat_interleave(torch.tensor(_cu(s["news"])[:-1]), torch.tensor(s["news"]))
            s["positions"] = (c["at"] + torch.arange(T) - first).to(torch.int32).cuda()
            s["freq"] = _frequencies(c)
            s["lengths_out"] = torch.zeros((B, hk), dtype=torch.int32, device="cuda")
        rows = rows.clamp(min=0)
        s["lengths"] = rows.to(torch.int32).contiguous()
        if c["op"] == "attend" and c["weights"]:
            s["weights"] = torch.rand((B, hk, s["capacity"]), generator=g, device="cuda")
            s["weights_out"] = torch.zeros_like(s["weights"])
        if c["op"] == "attend":
            s["lse"] = torch.zeros((B, hq, c["new"]), device="cuda")
        if c["op"] == "evict":
            # a few rows draw most of the attention; rows have changed places in earlier evictions
            s["weights"] = torch.exp(2.0 * torch.randn((B, hk, s["capacity"]), generator=g, device="cuda"))
            s["positions"] = torch.argsort(torch.rand((B, hk, s["capacity"]), generator=g, device="cuda"), dim=-1).to(torch.int32)
            s["weights_out"], s["positions_out"] = torch.zeros_like(s["weights"]), torch.zeros_like(s["positions"])
            s["lengths_out"] = torch.zeros_like(s["lengths"])
    if own:
        s["call"] = _handle(c, s)
    return s


def _handle(c, s):
    """The call with its arguments laid out once, as an engine keeps one per layer."""
    from paper_2503_17922_b200 import binding as wkv
    shape = dict(dtype=c["dtype"], batch=c["batch"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], head_dim=c["d"])
    rope = None
    if c["op"] in ("rotate", "append"):
        rope = wkv.Rope(c["rot"], _BASE, order=c["order"], scaling=c["scaling"], factor=_FACTOR, original_length=_ORIGINAL,
                        low=_LOW, high=_HIGH)
    if c["op"] in ("prompt", "rotate"):
        prob = wkv.Problem(l_obs=c.get("alpha", 1), window=8, task=0, top_p=0, max_seqlen=c["n"], budgets=[c["n"]] * c["batch"],
                           cu_seqlens=s["cu"], kv_layout=c["layout"], **shape)
        if c["op"] == "rotate":
            return wkv.prepare_rotate_prompt(prob, rope, s["q"], s["k"], s["q_out"], s["k_out"])
        return wkv.prepare_attend_prompt(prob, s["q"], s["k"], s["v"], s["q_out"], lse=s["lse"], lse_obs=s["lse_obs"])
    cache = wkv.PagedCache(page_size=c["page"], num_pages=s["num_pages"], block_table=s["table"], max_new=c.get("new", 1),
                           cu_new=s.get("cu"), layout=c["layout"], **shape)
    if c["op"] == "append":
        return wkv.prepare_append_kv_paged(cache, s["k"], s["v"], s["lengths"], s["k_pools"][0], s["v_pools"][0], q=s["q"],
                                           q_out=s["q_out"], positions=s["positions"], rope=rope, lengths_out=s["lengths_out"])
    if c["op"] == "attend":
        return wkv.prepare_attend_paged(cache, s["q"], s["k_pools"][0], s["v_pools"][0], s["lengths"], s["q_out"],
                                        cache.alloc_workspace(), lse=s["lse"], weights_in=s.get("weights"),
                                        weights_out=s.get("weights_out"))
    return wkv.prepare_evict_kv_paged(cache, s["k_pools"], s["v_pools"], s["weights"], s["positions"], s["lengths"], c["budget"],
                                      c["recent"], s["weights_out"], s["positions_out"], s["lengths_out"],
                                      cache.alloc_workspace())


# ---- one pass ----------------------------------------------------------------------------------
def run(state):
    s, op = state, state["case"]["op"]
    if own:
        s["call"].run()
        if op == "prompt":
            return {"out": s["q_out"], "lse": s["lse"], "lse_obs": s["lse_obs"]}
        if op == "rotate":
            return {"q": s["q_out"], "k": s["k_out"]}
        if op == "append":
            return {"q": s["q_out"], "k_pool": s["k_pools"][0], "v_pool": s["v_pools"][0], "lengths": s["lengths_out"]}
        if op == "attend":
            return {"out": s["q_out"], "lse": s["lse"], "weights": s.get("weights_out")}
        return {"k_pools": s["k_pools"], "v_pools": s["v_pools"], "weights": s["weights_out"], "positions": s["positions_out"],
                "lengths": s["lengths_out"]}
    return {"prompt": _prompt, "rotate": _rotate, "append": _append, "attend": _attend, "evict": _evict}[op](s)


def _padded(x, lens, cu, most):
    """Packed [T, h, d] -> [B, h, most, d]; rows behind a sequence's last are repetitions of some row (masked or unused)."""
    at = torch.tensor(cu[:-1], device=x.device).view(-1, 1) + torch.arange(most, device=x.device).view(1, -1)
    return x[at.clamp(max=x.shape[0] - 1)].transpose(1, 2)


def _packed(x, lens):
    """[B, h, most, d] -> packed [T, h, d]."""
    there = torch.arange(x.shape[2], device=x.device).view(1, -1) < torch.tensor(lens, device=x.device).view(-1, 1)
    return x.transpose(1, 2)[there]


def _softmax_rows(q, k, v, visible):
    """q [B, hk, G, M, d] over k, v [B, hk, N, d]; query m of head h sees the first visible[B, hk, M] rows.
    Returns the output, the log-sum-exp and the probabilities; a row that sees nothing has output 0."""
    x = torch.matmul(q.flatten(2, 3), k.transpose(-1, -2)).unflatten(2, q.shape[2:4]) / math.sqrt(q.shape[-1])
    hidden = torch.arange(k.shape[2], device=k.device) >= visible.unsqueeze(-1)
    x.masked_fill_(hidden.unsqueeze(2), float("-inf"))
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    p = x.sub_(top).exp_()
    z = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, q.shape[2:4]) / torch.where(z == 0, torch.ones_like(z), z)
    return out, (z.log() + top).squeeze(-1), p, z


def _prompt(s):
    c = s["case"]
    B, n, hk, G = c["batch"], c["n"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    q, k, v = s["q"], s["k"], s["v"]
    if c["ragged"]:
        q, k, v = (_padded(x, s["lens"], s["cu"], n) for x in (q, k, v))
    q, k, v = q.float().unflatten(1, (hk, G)), k.float(), v.float()
    lens = torch.tensor(s["lens"], device="cuda")
    out, lse = torch.empty_like(q), torch.empty(q.shape[:-1], device="cuda")
    # the scores of all rows at once would not fit: some hundred million at a time
    step = max(1, 2 ** 29 // (B * c["q_heads"] * n))
    for lo in range(0, n, step):
        hi = min(n, lo + step)
        visible = (torch.arange(lo, hi, device="cuda") + 1).expand(B, hk, hi - lo)
        out[:, :, :, lo:hi], lse[:, :, :, lo:hi], _, _ = _softmax_rows(q[:, :, :, lo:hi], k[:, :, :hi], v[:, :, :hi], visible)
    out, lse = out.flatten(1, 2), lse.flatten(1, 2)
    at = lens.view(B, 1, 1) - c["alpha"] + torch.arange(c["alpha"], device="cuda")
    lse_obs = torch.where(at < 0, torch.full_like(lse[:, :, :1], float("-inf")), lse.gather(2, at.clamp(min=0).expand(B, c["q_heads"], -1)))
    lse = torch.where(torch.arange(n, device="cuda") < lens.view(B, 1, 1), lse, torch.zeros_like(lse))
    out = out.to(_dtype(c))
    return {"out": _packed(out, s["lens"]) if c["ragged"] else out, "lse": lse, "lse_obs": lse_obs}


def _turned(x, angle, c):
    """x [..., d] with its first `rot` dimensions rotated by `angle` [..., rot / 2] (64 bits)."""
    rot = c["rot"]
    cos, sin = angle.cos().float(), angle.sin().float()
    y = x.float()
    if c["order"] == "half":
        a, b = y[..., : rot // 2], y[..., rot // 2: rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _rotate(s):
    c = s["case"]
    if c["ragged"]:
        at = torch.cat([torch.arange(n) for n in s["lens"]]).cuda().view(-1, 1)       # [T, 1, .]
    else:
        at = torch.arange(c["n"], device="cuda")                                      # [n, .]
    angle = at.double().unsqueeze(-1) * s["freq"].cuda()
    return {"q": _turned(s["q"], angle, c), "k": _turned(s["k"], angle, c)}


def _sequence_of(news):
    return torch.repeat_interleave(torch.arange(len(news)), torch.tensor(news)).cuda()


def _tokens(x, ragged):
    """New tokens as [T, h, d], packed or dense."""
    return x if ragged else x.transpose(1, 2).flatten(0, 1)


def _places(s, b, h, row):
    """Index of row `row` of unit (b, h) in a pool."""
    c = s["case"]
    page, slot = s["table"][b, row // c["page"]].long(), row % c["page"]
    return (page, h, slot) if c["layout"] == "phsd" else (page, slot, h)


def _append(s):
    c = s["case"]
    B, hk = c["batch"], c["kv_heads"]
    news = torch.tensor(s["news"], device="cuda")
    angle = s["positions"].double().view(-1, 1, 1) * s["freq"].cuda()
    q = _turned(_tokens(s["q"], c["ragged"]), angle, c)
    if not c["ragged"]:
        q = q.unflatten(0, (B, c["new"])).transpose(1, 2)
    b = _sequence_of(s["news"]).view(-1, 1)
    h = torch.arange(hk, device="cuda").view(1, -1)
    nth = (torch.arange(b.shape[0], device="cuda") - (news.cumsum(0) - news)[b.view(-1)]).view(-1, 1)
    at = _places(s, b, h, s["lengths"].long()[b, h] + nth)
    s["k_pools"][0][at] = _turned(_tokens(s["k"], c["ragged"]), angle, c)
    s["v_pools"][0][at] = _tokens(s["v"], c["ragged"])
    return {"q": q, "k_pool": s["k_pools"][0], "v_pool": s["v_pools"][0], "lengths": s["lengths"] + news.view(-1, 1).to(torch.int32)}


def _cached(s, pool):
    """The rows of every unit in order, [B, hk, capacity, d] in 32 bits."""
    x = pool[s["table"].long()]                                                       # [B, pages, ., ., d]
    x = x.transpose(1, 2) if s["case"]["layout"] == "phsd" else x.permute(0, 3, 1, 2, 4)
    return x.flatten(2, 3).float()


def _attend(s):
    c = s["case"]
    B, hk, G, new = c["batch"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["new"]
    q = _padded(s["q"], s["news"], s["cu"], new) if c["ragged"] else s["q"]
    k, v = _cached(s, s["k_pools"][0])[:, :, : c["n"]], _cached(s, s["v_pools"][0])[:, :, : c["n"]]
    news = torch.tensor(s["news"], device="cuda").view(B, 1, 1)
    nth = torch.arange(new, device="cuda").view(1, 1, -1)
    visible = torch.where(nth < news, s["lengths"].unsqueeze(-1) - news + nth + 1, torch.zeros_like(nth))
    out, lse, p, z = _softmax_rows(q.float().unflatten(1, (hk, G)), k, v, visible)
    lse = torch.where(nth < news, lse.flatten(1, 2), torch.zeros_like(lse.flatten(1, 2)))
    out = out.flatten(1, 2).to(_dtype(c))
    weights = None
    if c["weights"]:
        # a sum of few positive terms beside a term of a thousand cached rows' size: 64 bits for the column sums
        mine = p.div_(torch.where(z == 0, torch.ones_like(z), z)).sum((2, 3), dtype=torch.float64)
        there = torch.arange(c["n"], device="cuda") < s["lengths"].unsqueeze(-1)
        weights = torch.zeros_like(s["weights"])
        weights[:, :, : c["n"]] = torch.where(there, s["weights"][:, :, : c["n"]] + mine, torch.zeros_like(mine)).float()
    return {"out": _packed(out, s["news"]) if c["ragged"] else out, "lse": lse, "weights": weights}


def _evict(s):
    c = s["case"]
    lens = s["lengths"].long().unsqueeze(-1)
    B, hk, cap = s["weights"].shape
    row = torch.arange(cap, device="cuda").expand(B, hk, cap)
    there = row < lens
    keep = lens.clamp(max=c["budget"])
    newest = torch.where(there, s["positions"], torch.full_like(s["positions"], -1)).amax(-1, keepdim=True)
    first = there & (s["positions"] > newest - c["recent"])
    # rows by (recent first, weight from high to low, row from low to high); those that are not there last
    order = torch.sort(torch.where(there, s["weights"], torch.full_like(s["weights"], -1.0)), dim=-1, descending=True, stable=True).indices
    rank_of = first.gather(-1, order).long() * 2 + there.gather(-1, order).long()
    order = order.gather(-1, torch.sort(rank_of, dim=-1, descending=True, stable=True).indices)
    stays = torch.zeros_like(there).scatter_(-1, order, row < keep)
    # the i-th row that leaves in front of row `keep` takes the i-th that stays behind it
    hole, fill = ~stays & (row < keep), stays & (row >= keep)
    b, h, to = hole.nonzero(as_tuple=True)
    _, _, source = fill.nonzero(as_tuple=True)
    weights = torch.where(row < keep, s["weights"], torch.zeros_like(s["weights"]))
    positions = torch.where(row < keep, s["positions"], torch.zeros_like(s["positions"]))
    weights[b, h, to], positions[b, h, to] = s["weights"][b, h, source], s["positions"][b, h, source]
    at, come = _places(s, b, h, to), _places(s, b, h, source)
    for pool in s["k_pools"] + s["v_pools"]:
        pool[at] = pool[come]
    return {"k_pools": s["k_pools"], "v_pools": s["v_pools"], "weights": weights, "positions": positions,
            "lengths": keep.squeeze(-1).to(torch.int32)}


# ---- the definition in 64 bits ------------------------------------------------------------------
def _exact_rows(q, keys, values, limits):
    """softmax(q k / sqrt(d)) v of the rows of one head, 64 bits; row i sees the first limits[i] keys."""
    out, lse = torch.zeros_like(q), torch.full(q.shape[:1], float("-inf"), dtype=torch.float64, device=q.device)
    received = torch.zeros(keys.shape[0], dtype=torch.float64, device=q.device)
    step = max(1, 2 ** 27 // max(1, keys.shape[0]))
    for lo in range(0, q.shape[0], step):
        lim = limits[lo:lo + step]
        most = int(lim.max())
        if most <= 0:
            continue
        x = q[lo:lo + step] @ keys[:most].T * (q.shape[1] ** -0.5)
        x[torch.arange(most, device=q.device)[None, :] >= lim[:, None]] = float("-inf")
        lse[lo:lo + step] = torch.logsumexp(x, 1)
        p = torch.exp(x - lse[lo:lo + step, None])
        p[lim <= 0] = 0.0
        out[lo:lo + step] = p @ values[:most]
        received[:most] += p.sum(0)
    return out, lse, received


def exact(case, seed):
    global own
    c, was = case, own
    own = False
    s = prepare(case, seed)
    own = was
    B, hq, hk, d = c["batch"], c["q_heads"], c["kv_heads"], c["d"]
    G = hq // hk
    f64 = torch.float64
    if c["op"] == "prompt":
        out = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
        lse, lse_obs = torch.zeros((B, hq, c["n"]), dtype=f64, device="cuda"), torch.full((B, hq, c["alpha"]), float("-inf"), dtype=f64, device="cuda")
        for b, n in enumerate(s["lens"]):
            for h in range(hq):
                part = (slice(s["cu"][b], s["cu"][b] + n), h) if c["ragged"] else (b, h)
                kv = part[:-1] + (h // G,)
                o, l, _ = _exact_rows(s["q"][part].double(), s["k"][kv].double(), s["v"][kv].double(),
                                      torch.arange(1, n + 1, device="cuda"))
                out[part], lse[b, h, :n] = o, l
                m = min(n, c["alpha"])
                lse_obs[b, h, c["alpha"] - m:] = l[n - m:]
        return {"out": out, "lse": lse, "lse_obs": lse_obs}

    def rotated(x, positions):       # x [tokens, heads, d], one position per token
        y = x.double()
        z = y.clone()
        for i in range(c["rot"] // 2):
            j, k = (i, i + c["rot"] // 2) if c["order"] == "half" else (2 * i, 2 * i + 1)
            a = (positions.double() * float(s["freq"][i]))[:, None]
            z[..., j] = y[..., j] * torch.cos(a) - y[..., k] * torch.sin(a)
            z[..., k] = y[..., j] * torch.sin(a) + y[..., k] * torch.cos(a)
        return z

    if c["op"] == "rotate":
        got = {}
        for name in ("q", "k"):
            z = torch.empty(s[name].shape, dtype=f64, device="cuda")
            for b, n in enumerate(s["lens"]):
                if c["ragged"]:
                    at = slice(s["cu"][b], s["cu"][b] + n)
                    z[at] = rotated(s[name][at], torch.arange(n, device="cuda"))
                else:
                    z[b] = rotated(s[name][b].transpose(0, 1), torch.arange(n, device="cuda")).transpose(0, 1)
            got[name] = z
        return got

    def rows_of(pool, b, h, count):
        pages = s["table"][b, : (count + c["page"] - 1) // c["page"]].long()
        x = pool[pages, h] if c["layout"] == "phsd" else pool[pages, :, h]
        return x.reshape(-1, d)[:count].double()

    if c["op"] == "attend":
        out = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
        lse = torch.zeros((B, hq, c["new"]), dtype=f64, device="cuda")
        weights = torch.zeros(s["weights"].shape, dtype=f64, device="cuda") if c["weights"] else None
        for b, m in enumerate(s["news"]):
            for h in range(hk):
                n = int(s["lengths"][b, h])
                keys, values = rows_of(s["k_pools"][0], b, h, n), rows_of(s["v_pools"][0], b, h, n)
                if c["weights"]:
                    weights[b, h, :n] = s["weights"][b, h, :n].double()
                for head in range(h * G, h * G + G):
                    part = (slice(s["cu"][b], s["cu"][b] + m), head) if c["ragged"] else (b, head)
                    o, l, r = _exact_rows(s["q"][part].double(), keys, values, torch.arange(n - m + 1, n + 1, device="cuda"))
                    out[part], lse[b, head, :m] = o, l
                    if c["weights"]:
                        weights[b, h, :n] += r
        return {"out": out, "lse": lse, "weights": weights}

    if c["op"] == "append":
        pools = [s["k_pools"][0].double(), s["v_pools"][0].double()]
        q = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
        first = 0
        for b, m in enumerate(s["news"]):
            at = slice(first, first + m)
            pos = s["positions"][at]
            first += m
            if c["ragged"]:
                q[at] = rotated(s["q"][at], pos)
                k, v = rotated(s["k"][at], pos), s["v"][at].double()
            else:
                q[b] = rotated(s["q"][b].transpose(0, 1), pos).transpose(0, 1)
                k, v = rotated(s["k"][b].transpose(0, 1), pos), s["v"][b].transpose(0, 1).double()
            for h in range(hk):
                row = int(s["lengths"][b, h]) + torch.arange(m, device="cuda")
                page, slot = s["table"][b][row // c["page"]].long(), row % c["page"]
                for pool, new in zip(pools, (k, v)):
                    (pool[:, h] if c["layout"] == "phsd" else pool[:, :, h])[page, slot] = new[:, h]
        return {"q": q, "k_pool": pools[0], "v_pool": pools[1], "lengths": None}
    # evict: rows are only moved; the weights' places are found here by sorting each unit on its own
    weights = torch.zeros(s["weights"].shape, dtype=f64, device="cuda")
    for b in range(B):
        for h in range(hk):
            n = int(s["lengths"][b, h])
            keep = min(n, c["budget"])
            w, pos = s["weights"][b, h, :n].cpu().tolist(), s["positions"][b, h, :n].cpu().tolist()
            newest = max(pos, default=0)
            stays = sorted(range(n), key=lambda r: (pos[r] <= newest - c["recent"], -w[r], r))[:keep]
            fill = iter(sorted(r for r in stays if r >= keep))
            held = set(stays)
            kept = [w[r] if r in held else w[next(fill)] for r in range(keep)]
            weights[b, h, :keep] = torch.tensor(kept, dtype=f64, device="cuda")
    return {"k_pools": None, "v_pools": None, "weights": weights, "positions": None, "lengths": None}
