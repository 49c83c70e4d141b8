"""GPU tests of drafts at the limits: a cache that has no rows left for a whole draft, batches without a token, and units whose work several blocks share;
each against a reference in 64 bits."""
import pytest
import torch

import cache8_util as cu
import operators_util as ou
from paper_2503_17922_b200 import binding as wkv
from test_gpu_cache8 import DT, Attend, cumulated, gen, name_of, randn, random_tree

pytestmark = pytest.mark.gpu


# ---- drafts that the cache has no rows for -----------------------------------------------------------
CUT = [
    # dtype, kind, hq, hk, d, page, pages of a sequence, layout, news, packed
    ("bf16", "plain", 4, 2, 128, 16, 6, "phsd", [5, 5, 5], False),
    ("bf16", "plain", 8, 2, 64, 8, 20, "pshd", [12, 7, 12], True),
    ("bf16", "plain", 4, 2, 128, 16, 20, "phsd", [40, 40, 33], True),
    ("bf16", "plain", 4, 2, 64, 6, 30, "phsd", [30, 30, 30], False),
    ("bf16", "e4m3", 4, 2, 128, 16, 6, "pshd", [5, 5, 5], False),
    ("bf16", "i8", 8, 2, 64, 16, 20, "phsd", [40, 40, 40], False),
    ("bf16", "e4m3", 4, 2, 256, 16, 9, "phsd", [17, 3, 40], True),
    ("f32", "plain", 4, 2, 64, 16, 9, "phsd", [7, 7, 7], False),
    ("f32", "plain", 4, 2, 128, 16, 9, "pshd", [40, 33, 1], True),
    ("f32", "i8", 4, 2, 80, 16, 9, "phsd", [20, 20, 20], False),
    ("bf16", "plain", 4, 2, 128, 16, 132, "phsd", [70, 64, 70], True),
    ("bf16", "i8", 8, 2, 96, 32, 70, "pshd", [40, 40, 40], False),
]


@pytest.mark.parametrize("case", CUT, ids=name_of)
def test_a_draft_that_the_cache_has_no_rows_for(case):
    """Units with room for the whole draft, exactly, for a part of it and for none of it: the dropped tokens are seen and kept by none, the others
    attend and are kept as ever, and no row in front of the draft changes."""
    dtype, kind, hq, hk, d, page, max_pages, layout, news, packed = case
    g, B, most, G, eight = gen(31), len(news), max(news), hq // hk, kind != "plain"
    c = cu.Cache8(g, kind, B, hk, d, page, max_pages, layout) if eight else ou.Cache(g, DT[dtype], B, hk, d, page, max_pages, layout, fill=55.0)
    cap = c.cap
    first = [[cap - news[0] - 9, cap - news[0]], [cap - (news[1] + 1) // 2, cap], [cap - 1, 3]]
    c.fill(g, first)
    cu_new = cumulated(news) if packed else None
    if eight:
        cache, (layer,) = c.describe(dtype, hq, most, cu_new)
        tensors = c.codes[0] + c.scales[0]
    else:
        cache = wkv.PagedCache(dtype=dtype, batch=B, n_q_heads=hq, n_kv_heads=hk, head_dim=d, page_size=page, num_pages=c.num_pages, block_table=c.table,
                               max_new=most, cu_new=cu_new, layout=layout)
        tensors = c.k + c.v
    q, k, v = (randn(g, *((sum(news), h, d) if packed else (B, h, most, d)), dtype=DT[dtype]) for h in (hq, hk, hk))
    parents = [random_tree(g, m, 0.1) for m in news]
    sees = [cu.tree_of(p) for p in parents]
    flat = torch.tensor([x for p in parents for x in p], dtype=torch.int32)
    flat = (flat if packed else flat.view(B, most)).cuda()
    masks = torch.zeros((*flat.shape, (most + 31) // 32), dtype=torch.int32, device="cuda")
    at = torch.zeros_like(flat)
    wkv.wkv_draft_masks(cache, flat, masks, torch.full((B,), 1000, dtype=torch.int32, device="cuda"), at)
    before = torch.tensor(first, dtype=torch.int32, device="cuda")
    grown = torch.full_like(before, 77)
    positions = torch.randint(0, 999, (B, hk, cap), generator=g).to(torch.int32).cuda()
    weights = torch.rand((B, hk, cap), generator=g).cuda()
    state = dict(positions=at, lengths_out=grown, row_positions=positions, row_weights=weights)
    if eight:
        wkv.wkv_append_kv_paged8(cache, layer, k, v, before, **state)
    else:
        wkv.wkv_append_kv_paged(cache, k, v, before, c.k[0], c.v[0], **state)
    out, lse, ws = torch.full_like(q, 77.0), torch.full((B, hq, most), 77.0, device="cuda"), cache.alloc_workspace()
    if eight:
        wkv.wkv_attend_paged8(cache, layer, q, grown, out, ws, lse=lse, draft=masks, before=before)
    else:
        wkv.wkv_attend_draft_paged(cache, masks, q, c.k[0], c.v[0], grown, out, ws, lse=lse, before=before)
    torch.cuda.synchronize()
    assert wkv.device_status(ws) == 0
    part = lambda t, b, h: t[cumulated(news)[b]:cumulated(news)[b + 1], h] if packed else t[b, h, : news[b]]
    rows = lambda kv, b, h, n: c.rows(0, kv, b, h, n) if eight else c.rows((c.v if kv else c.k)[0], b, h, n)
    for b, m in enumerate(news):
        for h in range(hk):
            L, n = first[b][h], min(first[b][h] + m, cap)
            assert int(grown[b, h]) == n
            (kk, _), (vv, _) = rows(0, b, h, n), rows(1, b, h, n)
            j = torch.arange(n)[None, :] - L
            seen = ((j < 0) | sees[b].gather(1, j.clamp(min=0).expand(m, n))).cuda()
            for head in range(h * G, h * G + G):
                ref, ref_lse, _, bd = cu.attention_seen(part(q, b, head), kk, vv, seen)
                ou.assert_close(part(out, b, head), ref, ou.output_bound(ref, bd, DT[dtype]), f"out {b} {head}")
                ou.assert_close(lse[b, head, :m], ref_lse, ou.lse_bound(ref_lse, bd), f"lse {b} {head}")
    # what is kept: the last token's path
    last = torch.tensor([m - 1 for m in news], dtype=torch.int32, device="cuda")
    held = [t.clone() for t in tensors]
    old_positions, old_weights, kept = positions.clone(), weights.clone(), torch.full_like(before, 77)
    if eight:
        wkv.wkv_keep_draft_paged8(cache, masks, [layer], last, grown, kept, positions, weights, before=before)
    else:
        wkv.wkv_keep_draft_paged(cache, masks, c.k, c.v, last, grown, kept, positions, weights, before=before)
    torch.cuda.synchronize()
    want = [t.clone() for t in held]
    want_positions, want_weights = old_positions.clone(), old_weights.clone()
    for b, m in enumerate(news):
        for h in range(hk):
            L, n = first[b][h], min(first[b][h] + m, cap)
            path = [j for j in range(m) if sees[b][m - 1, j] and L + j < n]
            assert int(kept[b, h]) == L + len(path)
            for x, j in enumerate(path):
                want_positions[b, h, L + x], want_weights[b, h, L + x] = old_positions[b, h, L + j], old_weights[b, h, L + j]
                src, dst = ((int(c.table[b, r // page]), r % page) for r in (L + j, L + x))
                for t, w in zip(held, want):
                    if t.dim() == 3 or layout == "phsd":
                        w[dst[0], h, dst[1]] = t[src[0], h, src[1]]
                    else:
                        w[dst[0], dst[1], h] = t[src[0], src[1], h]
    assert torch.equal(positions, want_positions) and torch.equal(weights, want_weights)
    for t, w in zip(tensors, want):
        assert torch.equal(t, w)


def test_rows_in_front_of_a_draft_are_limited_to_the_draft():
    """Entries that fit no draft count as the nearest that does: lengths less the tokens, or lengths."""
    g, m, n = gen(32), 20, 100
    c = ou.Cache(g, torch.bfloat16, 1, 1, 64, 16, 8)
    c.fill(g, [[n]])
    cache = wkv.PagedCache(dtype="bf16", batch=1, n_q_heads=2, n_kv_heads=1, head_dim=64, page_size=16, num_pages=c.num_pages, block_table=c.table, max_new=m)
    sees = cu.tree_of(random_tree(g, m))
    masks, q = cu.words_of(sees).view(1, m, 1).cuda(), randn(g, 1, 2, m, 64, dtype=torch.bfloat16)
    lengths, ws, outs = torch.full((1, 1), n, dtype=torch.int32, device="cuda"), cache.alloc_workspace(), {}
    for value in (None, -5, 0, n - m, n, n + 1, 2 ** 31 - 1):
        before = None if value is None else torch.full((1, 1), value, dtype=torch.int32, device="cuda")
        outs[value] = torch.full_like(q, 77.0)
        wkv.wkv_attend_draft_paged(cache, masks, q, c.k[0], c.v[0], lengths, outs[value], ws, before=before)
        kept = torch.zeros_like(lengths)
        wkv.wkv_keep_draft_paged(cache, masks, [c.k[0].clone()], None, torch.tensor([-1], dtype=torch.int32, device="cuda"), lengths, kept, before=before)
        assert int(kept) == (n if value is not None and value >= n else n - m)
    torch.cuda.synchronize()
    for value in (-5, 0, n - m):
        assert torch.equal(outs[value], outs[None])
    assert torch.equal(outs[n + 1], outs[n]) and torch.equal(outs[2 ** 31 - 1], outs[n])
    k, v = c.rows(c.k[0], 0, 0, n)[0], c.rows(c.v[0], 0, 0, n)[0]
    for head in range(2):
        ref, _, _, bd = cu.attention_seen(q[0, head], k, v, torch.ones((m, n), dtype=torch.bool, device="cuda"))
        ou.assert_close(outs[n][0, head], ref, ou.output_bound(ref, bd, torch.bfloat16), "all rows in front")


# ---- batches without a token -----------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["plain", "e4m3"])
@pytest.mark.parametrize("given", [False, True])
def test_a_step_in_which_no_sequence_drafts(kind, given):
    """Every call of a draft's step with packed tensors of no rows: nothing to attend or keep, and lengths stay."""
    g, d, lengths = gen(33), 64, [[20, 3], [0, 64]]
    c = cu.Cache8(g, kind, 2, 2, d, 16, 4) if kind != "plain" else ou.Cache(g, torch.bfloat16, 2, 2, d, 16, 4, fill=55.0)
    c.fill(g, lengths)
    if kind != "plain":
        cache, (layer,) = c.describe("bf16", 4, 5, [0, 0, 0])
        tensors = c.codes[0] + c.scales[0]
    else:
        cache = wkv.PagedCache(dtype="bf16", batch=2, n_q_heads=4, n_kv_heads=2, head_dim=d, page_size=16, num_pages=c.num_pages, block_table=c.table, max_new=5,
                               cu_new=[0, 0, 0])
        tensors = c.k + c.v
    held = [t.clone() for t in tensors]
    empty = lambda *s, dtype=torch.bfloat16: torch.zeros((0, *s), dtype=dtype, device="cuda")
    q, k, masks, ws = empty(4, d), empty(2, d), empty(1, dtype=torch.int32), cache.alloc_workspace()
    before = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    grown, kept = torch.full_like(before, 77), torch.full_like(before, 77)
    last, more = torch.tensor([-1, 0], dtype=torch.int32, device="cuda"), dict(before=before) if given else {}
    wkv.wkv_draft_masks(cache, empty(dtype=torch.int32), masks)
    if kind != "plain":
        wkv.wkv_append_kv_paged8(cache, layer, k, k, before, lengths_out=grown)
        wkv.wkv_attend_paged8(cache, layer, q, grown, q.clone(), ws, draft=masks, **more)
        wkv.wkv_keep_draft_paged8(cache, masks, [layer], last, grown, kept, **more)
    else:
        wkv.wkv_append_kv_paged(cache, k, k, before, c.k[0], c.v[0], lengths_out=grown)
        wkv.wkv_attend_draft_paged(cache, masks, q, c.k[0], c.v[0], grown, q.clone(), ws, **more)
        wkv.wkv_keep_draft_paged(cache, masks, c.k, c.v, last, grown, kept, **more)
    torch.cuda.synchronize()
    assert torch.equal(grown, before) and torch.equal(kept, before)
    for t, w in zip(tensors, held):
        assert torch.equal(t, w)


# ---- units whose work several blocks share -----------------------------------------------------------------
# The tensor-core kernel cuts its items (256 query rows of a unit) into pieces where a unit can have 2,048 rows, and joins them: with up to 128 items by
# one kernel, with more by another.  Everything here has more than 64 rows per unit, and so goes there.
MANY = [[2200 + h for h in range(8)]] + [[100 + 13 * b + h for h in range(8)] for b in range(15)] + [[33] * 8]
SHARED = [
    # dtype, kind, hq, hk, d, page, layout, lengths, news, packed, tree, hole
    ("bf16", "plain", 4, 1, 128, 16, "phsd", [[2300], [130], [70]], [70, 33, 70], True, True, (0, 3)),
    ("bf16", "plain", 6, 2, 80, 24, "pshd", [[2050, 2100], [60, 61]], [60, 25], True, False, None),
    ("bf16", "plain", 2, 2, 64, 8, "phsd", [[2500, 300]], [300], False, False, (0, 100)),
    ("bf16", "e4m3", 8, 2, 96, 64, "pshd", [[3000, 2990], [40, 40]], [40, 40], False, False, None),
    ("bf16", "i8", 4, 2, 80, 16, "phsd", [[2500, 2048], [700, 699]], [130, 100], True, True, (1, 2)),
    ("bf16", "e4m3", 4, 1, 128, 128, "phsd", [[5000]], [1024], False, True, None),
    ("bf16", "plain", 16, 8, 128, 16, "phsd", MANY, [40] + [33 + b % 8 for b in range(15)] + [33], True, True, (0, 60)),
    ("bf16", "i8", 16, 8, 96, 32, "pshd", MANY, [40] + [b % 41 for b in range(0, 150, 10)] + [33], True, False, None),
]


@pytest.mark.parametrize("case", SHARED, ids=lambda c: "-".join(map(str, c[:7])))
def test_shared_items_of_drafts(case):
    """Trees, and masks of any form; sequences with no rows in front of their draft, rows that see nothing, lengths of zero."""
    g, news, tree = gen(41), case[8], case[10]
    sees = [cu.tree_of(random_tree(g, m)) if tree else torch.rand((m, m), generator=g) < 0.3 for m in news]
    if not tree:
        for s in sees:
            s[:1] = False
    a = Attend(*case[:10], sees=sees, hole=case[11])
    units, pairs = len(news) * a.hk, -(-max(max(news), 1) // (2 * (128 // (a.hq // a.hk))))
    assert a.c.cap >= 2048 and max(news) * a.hq // a.hk > 64 and (units * pairs > 128) == (case[7] is MANY)
    a.run()
    a.check()
    first = a.out.clone()
    a.run()
    torch.cuda.synchronize()
    assert torch.equal(a.out, first)                                      # pieces are joined in an order of their own


@pytest.mark.parametrize("kind,d", [("plain", 128), ("plain", 80), ("e4m3", 128), ("i8", 96)])
@pytest.mark.parametrize("front", [True, False])
def test_shared_items_do_not_see_other_branches(kind, d, front):
    """NaN (plain: infinities too) in a token's row reaches its descendants and nobody else, in the pieces of a cut item as in a whole one."""
    new = 70
    n = 2300 if front else new
    parents = random_tree(gen(42), new, 0.3)
    sees = cu.tree_of(parents)
    a = Attend("bf16", kind, 4, 1, d, 16, "phsd", [[n], [2300]], [new, new], False, sees=[sees, sees])
    a.run()
    a.check()
    clean = a.out.clone()
    token = new // 3
    at = n - new + token
    if kind == "plain":
        a.c.slot(a.c.v[0], 0, 0, at)[3] = float("nan")
        a.c.slot(a.c.v[0], 0, 0, at)[5] = -float("inf")
    else:
        codes, scales, _ = a.c.raw(0, 1, 0, 0, n)
        if kind == "e4m3":
            codes[at, 3] = 0x7f
        else:
            scales[at] = 255
        a.c.put(0, 1, 0, 0, torch.arange(n), codes, scales)
    a.run()
    torch.cuda.synchronize()
    on = sees[:, token].cuda()
    assert torch.equal(a.out[0][:, ~on], clean[0][:, ~on]) and torch.equal(a.out[1], clean[1])
    assert torch.isnan(a.out[0][:, on][..., 3]).all() and not torch.isnan(clean).any()
    if kind == "plain":
        assert (a.out[0][:, on][..., 5] == -float("inf")).all()


@pytest.mark.parametrize("kind", ["plain", "e4m3"])
def test_shared_items_of_two_streams_and_a_captured_call(kind):
    """Two calls at once with workspaces of their own, and a captured one replayed on other inputs, give what each gives alone."""
    def make(seed):
        sees = [cu.tree_of(random_tree(gen(seed), 70)) for _ in range(2)]
        return Attend("bf16", kind, 8, 2, 128, 16, "phsd", [[2300, 2290], [300, 299]], [70, 70], False, sees=sees, seed=seed)
    a, b = make(1), make(2)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                x.run()
    a.check()
    b.check()
    want = b.out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    pools = (lambda x: x.c.k + x.c.v) if kind == "plain" else (lambda x: x.c.codes[0] + x.c.scales[0])
    for x, y in [(a.q, b.q), (a.masks, b.masks), (a.c.table, b.c.table)] + list(zip(pools(a), pools(b))):
        x.copy_(y)
    for _ in range(2):
        a.out.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want)
    del graph
