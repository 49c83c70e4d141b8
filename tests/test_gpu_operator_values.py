"""GPU tests of what infinities, NaN and rows without weight do in the attention kernels: the same in every one of them, whichever the
sizes lead to."""
import pytest
import torch

import operators_util as ou
from test_gpu_operators import Attend, INF, NAN, Prompt, tokens_of

pytestmark = pytest.mark.gpu

# A call over the paged cache for each kernel and each way of joining key splits
PAGED = {
    "tcgen05-shared-items": ("bf16", 8, 2, 128, 64, "phsd", [[4000, 3990]], [40], False),
    "tcgen05-shared-items-160": ("bf16", 32, 8, 128, 64, "phsd", [[2200] * 8] * 20, [9] * 20, False),
    "tcgen05": ("bf16", 8, 2, 128, 64, "phsd", [[1500, 1490]], [40], False),
    "warps-cluster": ("bf16", 8, 2, 128, 16, "phsd", [[992, 990]], [3], False),
    "warps-splits": ("bf16", 8, 2, 128, 64, "phsd", [[16000, 15990]], [3], False),
    "warps-many-rows": ("bf16", 8, 2, 128, 13, "phsd", [[1500, 1490]], [40], False),
    "fp32-cluster": ("f32", 4, 2, 64, 16, "phsd", [[700, 690]], [3], False),
    "fp32-splits": ("f32", 4, 2, 64, 16, "phsd", [[9000, 8990]], [3], False),
    "fp32-many-rows": ("f32", 4, 2, 64, 16, "phsd", [[1500, 1490]], [40], False),
}
# ... and a prompt (n tokens)
PROMPTS = {
    "tcgen05": ("bf16", 8, 2, 128, [700]),
    "tcgen05-64": ("bf16", 4, 2, 64, [700]),
    "warps": ("bf16", 4, 2, 128, [100]),
    "fp32-one-tile": ("f32", 4, 2, 64, [40]),
    "fp32-cluster": ("f32", 4, 2, 64, [300]),
}
paged_calls = pytest.mark.parametrize("name", PAGED)
prompts = pytest.mark.parametrize("name", PROMPTS)


def unit_rows(a, h=0):
    return min(int(a.lengths[0, h]), a.c.cap)


def set_rows(a, pool, h, rows, value, column=slice(None)):
    """Elements of rows of unit (0, h)."""
    pages, slots = a.c.table[0].long()[rows // a.c.page], (rows % a.c.page).cuda()
    pool[pages, h, slots, column] = value


def same_bits(x, y):
    kind = {2: torch.int16, 4: torch.int32}[x.element_size()]
    return torch.equal(x.contiguous().view(kind), y.contiguous().view(kind))


# ---- NaN among the queries and the keys ------------------------------------------------------
@paged_calls
def test_a_nan_query_gives_nan(name):
    """Its own row alone, and not the 0 and -infinity of a query that has nothing to attend to."""
    a = Attend(*PAGED[name])
    a.run(weights=False)
    torch.cuda.synchronize()
    out, lse = a.out.clone(), a.lse.clone()
    i = a.max_new // 2
    a.q[0, 1, i, 5] = NAN
    a.run(weights=False)
    torch.cuda.synchronize()
    assert torch.isnan(a.out[0, 1, i]).all() and torch.isnan(a.lse[0, 1, i])
    a.out[0, 1, i], a.lse[0, 1, i] = out[0, 1, i], lse[0, 1, i]
    assert same_bits(a.out, out) and same_bits(a.lse, lse)


@paged_calls
@pytest.mark.parametrize("part", ["first", "middle"])
def test_a_stretch_of_nan_keys_gives_nan(name, part):
    """NaN in all keys of a stretch of whole key tiles, all that some blocks have: every query that sees them is NaN."""
    a = Attend(*PAGED[name])
    n = unit_rows(a)
    a.run(weights=False)
    torch.cuda.synchronize()
    out, lse = a.out.clone(), a.lse.clone()
    first = 0 if part == "first" else n // 4 // 128 * 128
    rows = torch.arange(first, first + n // 3 // 128 * 128)
    set_rows(a, a.c.k[0], 0, rows, NAN)
    a.run(weights=False)
    torch.cuda.synchronize()
    G = a.hq // a.hk
    assert torch.isnan(a.out[0, :G]).all() and torch.isnan(a.lse[0, :G]).all()
    a.out[0, :G], a.lse[0, :G] = out[0, :G], lse[0, :G]
    assert same_bits(a.out, out) and same_bits(a.lse, lse)


# ---- infinities among values that are seen --------------------------------------------------------
@paged_calls
def test_an_infinity_in_a_row_of_tiny_weight_counts(name):
    """The first half's logits are so low that their weights are 0 in fp32: an infinity or NaN among their values still leaves one (0 times it
    is NaN), wherever the keys are split."""
    a = Attend(*PAGED[name])
    n, G, d = unit_rows(a), a.hq // a.hk, a.c.d
    a.q[:] = a.q.sign() * 0.5 + 1.0                                  # 0.5 or 1.5
    set_rows(a, a.c.k[0], 0, torch.arange(0, n // 2), -32.0)         # logits of -16 sqrt(d) and below, those of the others of the order of 1
    a.run()
    torch.cuda.synchronize()
    out, lse, w = a.out.clone(), a.lse.clone(), a.w_out.clone()
    assert torch.isfinite(out).all()
    set_rows(a, a.c.v[0], 0, torch.tensor([5]), INF, 3)
    set_rows(a, a.c.v[0], 0, torch.tensor([n // 4]), -INF, 4)
    set_rows(a, a.c.v[0], 0, torch.tensor([n // 2 - 1]), NAN, 6)
    a.run()
    torch.cuda.synchronize()
    assert not torch.isfinite(a.out[0, :G][..., [3, 4]]).any() and torch.isnan(a.out[0, :G, :, 6]).all()
    for c in (3, 4, 6):
        a.out[0, :G, :, c] = out[0, :G, :, c]
    assert same_bits(a.out, out) and same_bits(a.lse, lse) and same_bits(a.w_out, w)


@prompts
def test_an_infinity_in_a_prompt_row_of_tiny_weight_counts(name):
    p = Prompt(*PROMPTS[name])
    n = p.lens[0]
    p.q[:] = p.q.sign() * 0.5 + 1.0
    for row in (5, 17):
        p.k[0, 0, row] = -32.0
    p.run()
    torch.cuda.synchronize()
    out, G = p.out.clone(), p.hq // p.hk
    assert torch.isfinite(out).all()
    p.v[0, 0, 5, 3], p.v[0, 0, 17, 4] = INF, NAN
    p.run()
    torch.cuda.synchronize()
    assert not torch.isfinite(p.out[0, :G, 5:, 3]).any() and torch.isnan(p.out[0, :G, 17:, 4]).all()
    assert same_bits(p.out[0, :G, :5], out[0, :G, :5]) and same_bits(p.out[0, :G, :17, 4], out[0, :G, :17, 4])
    rest = [c for c in range(p.d) if c not in (3, 4)]
    assert same_bits(p.out[0, :G][..., rest], out[0, :G][..., rest]) and same_bits(p.out[0, G:], out[0, G:])


# ---- rows whose logits are all -infinity --------------------------------------------------------------
BELOW = 3.0e38               # times 3e4: beyond fp32, in whatever order the products are summed


@prompts
def test_a_prompt_row_of_logits_minus_infinity_is_zero(name):
    """No weight anywhere: 0 and -infinity, as for a row that has nothing to attend to."""
    p = Prompt(*PROMPTS[name])
    n, G = p.lens[0], p.hq // p.hk
    p.k[0, 0, :, 0], p.q[0, :G, :, 0] = -BELOW, 0.0
    p.run()
    torch.cuda.synchronize()
    out, lse = p.out.clone(), p.lse.clone()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    rows = [0, n // 2, n - 1]
    for i in rows:
        p.q[0, 0, i, 0] = 3.0e4
    p.run()
    torch.cuda.synchronize()
    for i in rows:
        assert (p.out[0, 0, i] == 0).all() and p.lse[0, 0, i] == -INF
        p.out[0, 0, i], p.lse[0, 0, i] = out[0, 0, i], lse[0, 0, i]
    assert same_bits(p.out, out) and same_bits(p.lse, lse)


@paged_calls
def test_a_query_of_logits_minus_infinity_is_zero(name):
    a = Attend(*PAGED[name])
    n, G = unit_rows(a), a.hq // a.hk
    set_rows(a, a.c.k[0], 0, torch.arange(n), -BELOW, 0)
    a.q[0, :G, :, 0] = 0.0
    a.run(weights=False)
    torch.cuda.synchronize()
    out, lse = a.out.clone(), a.lse.clone()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    i = a.max_new // 2
    a.q[0, 1, i, 0] = 3.0e4
    a.run(weights=False)
    torch.cuda.synchronize()
    assert (a.out[0, 1, i] == 0).all() and a.lse[0, 1, i] == -INF
    a.out[0, 1, i], a.lse[0, 1, i] = out[0, 1, i], lse[0, 1, i]
    assert same_bits(a.out, out) and same_bits(a.lse, lse)


@paged_calls
def test_a_query_of_logits_minus_infinity_leaves_no_weight(name):
    """The weights are those of the other queries."""
    a = Attend(*PAGED[name])
    n, G, m = unit_rows(a), a.hq // a.hk, a.max_new
    set_rows(a, a.c.k[0], 0, torch.arange(n), -BELOW, 0)
    a.q[0, :G, :, 0] = 0.0
    i = m // 2
    k, ok = a.c.rows(a.c.k[0], 0, 0, n)
    v, _ = a.c.rows(a.c.v[0], 0, 0, n)
    others = torch.tensor([g * m + j for g in range(G) for j in range(m) if (g, j) != (1, i)], device="cuda")
    qs = tokens_of(a.q, 0, a.news, a.packed)[:, :G].transpose(0, 1).reshape(G * m, -1)[others]
    _, _, p, bd = ou.attention(qs, k, v, torch.arange(n - m + 1, n + 1, device="cuda").repeat(G)[others], ok)
    a.q[0, 1, i, 0] = 3.0e4
    a.run()
    torch.cuda.synchronize()
    assert (a.out[0, 1, i] == 0).all() and a.lse[0, 1, i] == -INF
    want = a.w_in[0, 0, :n].double() + p.sum(0)
    bound = (bd["factor"][:, None] * p).sum(0) + G * m * ou.U * p.sum(0) + 2 * ou.U * want + 1e-37        # as in Attend.check
    ou.assert_close(a.w_out[0, 0, :n], want, bound, "weights")


@paged_calls
def test_a_nan_query_leaves_weights_alone_that_it_does_not_see(name):
    """Rows behind a query, and rows without a page, get nothing from it, NaN or not."""
    a = Attend(*PAGED[name])
    n, m = unit_rows(a), a.max_new
    a.c.table[0, 2] = -1
    a.run()
    torch.cuda.synchronize()
    clean = a.w_out.clone()
    missing = slice(2 * a.c.page, 3 * a.c.page)
    assert torch.isfinite(clean).all() and same_bits(clean[0, 0, missing], a.w_in[0, 0, missing])
    i = m // 2
    a.q[0, 1, i, 5] = NAN
    a.run()
    torch.cuda.synchronize()
    seen = n - m + i + 1
    assert same_bits(a.w_out[0, 0, seen:], clean[0, 0, seen:]) and same_bits(a.w_out[0, 0, missing], clean[0, 0, missing])
    rows = torch.arange(seen, device="cuda")
    assert torch.isnan(a.w_out[0, 0, :seen][(rows < missing.start) | (rows >= missing.stop)]).all()
    assert same_bits(a.w_out[0, 1:], clean[0, 1:])


# ---- many sequences --------------------------------------------------------------------------------
def test_row_state_of_many_sequences():
    """More (sequence, KV head) pairs than a grid's second dimension has room for."""
    from paper_2503_17922_b200 import binding as wkv
    B, H, n, alpha, window = 35000, 2, 12, 4, 4
    prob = wkv.Problem(dtype="bf16", batch=B, n_q_heads=2, n_kv_heads=H, head_dim=64, l_obs=alpha, window=window, task=0, top_p=0, max_seqlen=n,
                       budgets=[8] * B)
    idx = torch.randint(0, 2, (B, H, 1), generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()
    scores = torch.rand((B, H, n - alpha), device="cuda")
    positions = torch.full((B, H, 10), -1, dtype=torch.int32, device="cuda")
    weights = torch.full((B, H, 10), -1.0, device="cuda")
    wkv.wkv_seed_rows(prob, idx, scores, positions, weights)
    torch.cuda.synchronize()
    review = idx * window + torch.arange(window, dtype=torch.int32, device="cuda")
    assert torch.equal(positions[..., :4], review) and (positions[..., 4:8] == torch.arange(8, 12, device="cuda")).all() and (positions[..., 8:] == -1).all()
    assert torch.equal(weights[..., :4], scores.gather(-1, review.long())) and (weights[..., 4:8] == 0).all() and (weights[..., 8:] == -1).all()


# ---- strides that are not looked at -------------------------------------------------------------------
def test_the_batch_stride_of_packed_tensors_is_not_used():
    import ctypes
    from paper_2503_17922_b200 import binding as wkv
    L, stream = wkv.lib(), torch.cuda.current_stream().cuda_stream

    def st(t):
        return (ctypes.c_int64 * 3)(-5, t.stride(1), t.stride(0))
    p = Prompt("bf16", 4, 2, 64, [130, 70], "packed", 4)
    p.run()
    rope, turned, want_turned = wkv.Rope(64), torch.empty_like(p.q), torch.empty_like(p.q)
    wkv.wkv_rotate_prompt(p.prob, rope, p.q, None, want_turned, None)
    torch.cuda.synchronize()
    want = p.out.clone()
    p.out.fill_(77.0)
    s = ctypes.byref(p.prob.shape)
    assert L.wkv_attend_prompt(s, p.q.data_ptr(), st(p.q), p.k.data_ptr(), p.v.data_ptr(), p.out.data_ptr(), st(p.out), None, None, None, stream) == 0
    assert L.wkv_rotate_prompt(s, ctypes.byref(rope.struct), p.q.data_ptr(), turned.data_ptr(), st(p.q), None, None, None, stream) == 0
    torch.cuda.synchronize()
    assert same_bits(p.out, want) and same_bits(turned, want_turned)

    a = Attend("bf16", 4, 2, 64, 16, "phsd", [[80, 80], [60, 60]], [3, 4], True)
    a.run(weights=False)
    torch.cuda.synchronize()
    want, n = a.out.clone(), a.lengths.cuda()
    a.out.fill_(77.0)
    assert L.wkv_attend_paged(ctypes.byref(a.cache.shape), a.q.data_ptr(), st(a.q), a.c.k[0].data_ptr(), a.c.v[0].data_ptr(), n.data_ptr(),
                              a.out.data_ptr(), st(a.out), None, None, None, a.ws.data_ptr(), a.ws.numel(), stream) == 0
    torch.cuda.synchronize()
    assert same_bits(a.out, want)
    k, v = a.q[:, :2].contiguous(), a.q[:, 2:].contiguous()
    pools = []
    for strides in (None, st(k)):
        kp, vp, n1 = torch.zeros_like(a.c.k[0]), torch.zeros_like(a.c.k[0]), torch.zeros_like(n)
        if strides is None:
            wkv.wkv_append_kv_paged(a.cache, k, v, n, kp, vp, lengths_out=n1)
        else:
            assert L.wkv_append_kv_paged(ctypes.byref(a.cache.shape), None, k.data_ptr(), v.data_ptr(), strides, None, None, None, None, n.data_ptr(),
                                         kp.data_ptr(), vp.data_ptr(), n1.data_ptr(), None, None, stream) == 0
        torch.cuda.synchronize()
        pools.append((kp, vp, n1))
    assert all(same_bits(x, y) for x, y in zip(*pools))
