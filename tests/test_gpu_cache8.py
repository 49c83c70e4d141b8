"""GPU tests of the norms with rotary positions, the 8-bit cache and the drafts, each against a reference in 64 bits.  What a call must leave alone
is filled beforehand and looked at."""
import numpy as np
import pytest
import torch

import cache8_util as cu
import operators_util as ou
from paper_2503_17922_b200 import binding as wkv

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
INF, NAN = float("inf"), float("nan")


def gen(seed=1):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g).to(dtype).cuda()


def cumulated(lens):
    return np.concatenate([[0], np.cumsum(lens)]).tolist()


def problem(dtype, hq, hk, d, lens, layout, alpha=4, omega=8, budgets=None):
    n, B = max(lens), len(lens)
    return wkv.Problem(dtype=dtype, batch=B, n_q_heads=hq, n_kv_heads=hk, head_dim=d, l_obs=alpha, window=omega, task=0, top_p=0, max_seqlen=n,
                       budgets=budgets or [n] * B, cu_seqlens=cumulated(lens) if layout == "packed" else None,
                       kv_layout="bnhd" if layout == "packed" else layout)


# ---- norms with rotary positions ----------------------------------------------------------------
TURNS = [
    # dtype, d, norm, rot, order, axes, scale
    ("bf16", 128, True, 128, "half", 1, 1.0), ("bf16", 128, True, 128, "half", 3, 1.25), ("bf16", 128, True, 64, "interleaved", 2, 1.0),
    ("bf16", 128, True, 0, "half", 1, 1.0), ("bf16", 64, True, 24, "half", 2, 1.0), ("bf16", 80, True, 80, "half", 1, 1.0),
    ("bf16", 96, True, 62, "half", 3, 1.0), ("bf16", 128, False, 12, "half", 2, 1.0), ("bf16", 40, True, 6, "interleaved", 1, 1.0),
    ("bf16", 256, True, 256, "half", 1, 1.0), ("bf16", 256, True, 254, "half", 2, 1.0), ("bf16", 8, True, 2, "half", 1, 1.0),
    ("f32", 64, True, 64, "half", 1, 1.0), ("f32", 128, True, 96, "interleaved", 3, 0.5), ("f32", 4, True, 4, "half", 2, 1.0),
    ("f32", 256, True, 250, "half", 1, 1.0), ("f32", 20, False, 10, "half", 2, 1.0), ("f32", 256, True, 0, "half", 1, 1.0),
]


def turn_setup(dtype, d, norm, rot, order, axes, scale, tokens, g):
    rope = wkv.Rope(rot, 500000.0, order=order, scale=scale) if rot else None
    weights = [(1 + 0.3 * torch.randn(d, generator=g)).to(DT[dtype]).cuda() for _ in range(2)]
    axis = torch.randint(0, axes, (max(rot // 2, 1),), generator=g).tolist()
    positions = torch.randint(0, 2 ** 20, (axes, tokens), generator=g).to(torch.int32)
    return dict(rope=rope, norm=wkv.HeadNorm(*weights, eps=1e-5, offset=0.25) if norm else None,
                axes=wkv.RopeAxes(axis, axes) if rot and axes > 1 else None), weights, axis, positions


def check_turned(got, x, weight, case, axis, positions, what):
    dtype, d, norm, rot, order, axes, scale = case
    ref, big = cu.turned(x, weight, 1e-5 if norm else None, 0.25, positions, axis, ou.frequencies(rot, 500000.0) if rot else None, order, scale)
    r = ou.half_step(DT[dtype])
    ou.assert_close(got.cpu(), ref, cu.turned_bound(big, positions if rot else None, d, scale, norm) * (1 + r) + r * ref.abs(), what)


@pytest.mark.parametrize("case", TURNS, ids=lambda c: "-".join(map(str, c)))
def test_norm_rotate_prompt(case):
    dtype, d, norm, rot, order, axes, scale = case
    g, lens, hq, hk = gen(3), [1, 37, 80, 700], 6, 2
    tokens = sum(lens)
    prob = problem(dtype, hq, hk, d, lens, "packed")
    kw, weights, axis, positions = turn_setup(dtype, d, norm, rot, order, axes, scale, tokens, g)
    if not norm and not rot:
        return
    pos = positions.cuda() if axes > 1 else positions[0].cuda()
    if not rot:
        pos = None
    q, k = randn(g, tokens, hq, d, dtype=DT[dtype]) * 3, randn(g, tokens, hk, d, dtype=DT[dtype])
    q_out, k_out = torch.full_like(q, 77.0), torch.full_like(k, 77.0)
    wkv.wkv_norm_rotate_prompt(prob, q, k, q_out, k_out, positions=pos, **kw)
    torch.cuda.synchronize()
    check_turned(q_out, q, weights[0], case, axis, positions, "q")
    check_turned(k_out, k, weights[1], case, axis, positions, "k")
    # in place, and one tensor alone
    a, b = q.clone(), k.clone()
    wkv.wkv_norm_rotate_prompt(prob, a, None, a, None, positions=pos, **kw)
    wkv.wkv_norm_rotate_prompt(prob, None, b, None, b, positions=pos, **kw)
    torch.cuda.synchronize()
    assert torch.equal(a, q_out) and torch.equal(b, k_out)


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_norm_rotate_dense(layout):
    """Dense layouts with rows apart, places as positions, weights of one side alone, and none of one axis outside the table."""
    g, d, n = gen(4), 64, 50
    case = ("bf16", d, True, 32, "half", 1, 1.0)
    prob = problem("bf16", 4, 2, d, [n, n], layout)
    shape = (2, 4, n, d + 8) if layout == "bhnd" else (2, n, 4, d + 8)
    q = randn(g, *shape, dtype=torch.bfloat16)[..., :d]
    k = randn(g, *((2, 2, n, d) if layout == "bhnd" else (2, n, 2, d)), dtype=torch.bfloat16)
    if layout == "bnhd":
        q, k = q.transpose(1, 2), k.transpose(1, 2)
    q_out = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device="cuda")
    k_out = torch.empty_like(k)
    rope = wkv.Rope(32, 500000.0)
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(torch.bfloat16).cuda()
    wkv.wkv_norm_rotate_prompt(prob, q, k, q_out, k_out, norm=wkv.HeadNorm(w, None, eps=1e-5, offset=0.25), rope=rope)
    torch.cuda.synchronize()
    pos = torch.arange(n).view(1, -1)
    for b in range(2):
        check_turned(q_out[b].transpose(0, 1), q[b].transpose(0, 1), w, case, [0] * 16, pos, "q")
        check_turned(k_out[b].transpose(0, 1), k[b].transpose(0, 1), None, case, [0] * 16, pos, "k")
    # an axis that is none turns by nothing
    axes = wkv.RopeAxes([0] * 16, 1)
    axes.axis.fill_(5)
    wkv.wkv_norm_rotate_prompt(prob, q, None, q_out, None, rope=rope, axes=axes, positions=torch.full((1, 2, n), 9, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(q_out, q)


def test_rotation_without_norm_is_the_other_kernels():
    """One axis and no norm: the bits of wkv_rotate_prompt."""
    g, lens, d = gen(5), [60, 3], 128
    for dtype in ("bf16", "f32"):
        prob = problem(dtype, 4, 2, d, lens, "packed")
        q, k = randn(g, 63, 4, d, dtype=DT[dtype]), randn(g, 63, 2, d, dtype=DT[dtype])
        for rot, order in ((128, "half"), (36, "half"), (6, "half"), (64, "interleaved"), (6, "interleaved")):
            rope, outs = wkv.Rope(rot, 10000.0, order=order), [torch.full_like(x, 77.0) for x in (q, k, q, k)]
            wkv.wkv_rotate_prompt(prob, rope, q, k, outs[0], outs[1])
            wkv.wkv_norm_rotate_prompt(prob, q, k, outs[2], outs[3], rope=rope)
            torch.cuda.synchronize()
            assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


def test_norm_of_zeros_and_nan():
    prob = problem("bf16", 2, 2, 64, [4], "packed")
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    q[1, 0, 5], q[2, 1, 0] = NAN, INF
    out = torch.full_like(q, 77.0)
    wkv.wkv_norm_rotate_prompt(prob, q, None, out, None, norm=wkv.HeadNorm(eps=1e-6))
    torch.cuda.synchronize()
    assert torch.isnan(out[1, 0]).all() and torch.isnan(out[2, 1, 0])
    rest = out.clone()
    rest[1, 0], rest[2, 1] = 0, 0
    assert (rest == 0).all()


# ---- new tokens into the cache -------------------------------------------------------------------
def pool_row(cache, pool, b, h, row):
    page, slot = int(cache.table[b, row // cache.page]), row % cache.page
    return pool[page, h, slot] if cache.layout == "phsd" else pool[page, slot, h]


@pytest.mark.parametrize("dtype,layout,rot,order,axes", [("bf16", "phsd", 64, "half", 1), ("bf16", "pshd", 20, "interleaved", 2), ("f32", "phsd", 0, "half", 1)])
def test_norm_append(dtype, layout, rot, order, axes):
    """Rows of a plain cache are those of the prompt's call at the same positions; values are copies; what is beyond stays."""
    g, d, hq, hk, news = gen(6), 64, 4, 2, [3, 0, 5]
    c = ou.Cache(g, DT[dtype], 3, hk, d, 8, 3, layout, fill=55.0)
    c.table[2, 1] = -1
    T, cu_new = sum(news), cumulated(news)
    cache = wkv.PagedCache(dtype=dtype, batch=3, n_q_heads=hq, n_kv_heads=hk, head_dim=d, page_size=8, num_pages=c.num_pages, block_table=c.table,
                           max_new=5, cu_new=cu_new, layout=layout)
    kw, weights, axis, positions = turn_setup(dtype, d, True, rot, order, axes, 1.0, T, g)
    pos = positions.cuda() if axes > 1 else positions[0].cuda()
    q, k, v = (randn(g, T, h, d, dtype=DT[dtype]) for h in (hq, hk, hk))
    lengths = torch.tensor([[0, 7], [3, 3], [6, 22]], dtype=torch.int32, device="cuda")
    out, q_out = torch.full_like(lengths, 77), torch.full_like(q, 77.0)
    row_positions = torch.full((3, hk, c.cap), 77, dtype=torch.int32, device="cuda")
    row_weights = torch.full((3, hk, c.cap), 77.0, device="cuda")
    wkv.wkv_norm_append_kv_paged(cache, k, v, lengths, c.k[0], c.v[0], q=q, q_out=q_out, positions=pos, lengths_out=out, row_positions=row_positions,
                                 row_weights=row_weights, **kw)
    prob = problem(dtype, hq, hk, d, [T], "packed")
    q_ref, k_ref = torch.empty_like(q), torch.empty_like(k)
    wkv.wkv_norm_rotate_prompt(prob, q, k, q_ref, k_ref, positions=pos if rot else None, **kw)
    torch.cuda.synchronize()
    assert torch.equal(q_out, q_ref)
    written = [torch.zeros_like(c.k[0], dtype=torch.bool) for _ in range(2)]
    for b, m in enumerate(news):
        for h in range(hk):
            n = int(lengths[b, h])
            assert int(out[b, h]) == min(n + m, c.cap)
            for i in range(m):
                if n + i >= c.cap:
                    continue
                assert int(row_positions[b, h, n + i]) == int(positions[0, cu_new[b] + i]) and float(row_weights[b, h, n + i]) == 0
                if int(c.table[b, (n + i) // 8]) < 0:
                    continue
                assert torch.equal(pool_row(c, c.k[0], b, h, n + i), k_ref[cu_new[b] + i, h])
                assert torch.equal(pool_row(c, c.v[0], b, h, n + i), v[cu_new[b] + i, h])
                for w in written:
                    pool_row(c, w, b, h, n + i)[:] = True
            assert (row_positions[b, h, :n] == 77).all() and (row_positions[b, h, n + m:] == 77).all()
    assert (c.k[0][~written[0]] == 55).all() and (c.v[0][~written[1]] == 55).all()


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype,layout,d,rot,order", [("bf16", "phsd", 64, 64, "half"), ("f32", "pshd", 128, 52, "half"), ("bf16", "pshd", 80, 30, "interleaved"),
                                                      ("f32", "phsd", 16, 0, "half"), ("bf16", "phsd", 256, 254, "half")])
def test_append8(kind, dtype, layout, d, rot, order):
    """Codes and scales of the new rows.  Without norms a turned key is the number that the prompt's call gives in fp32, so its codes are that
    number's, bit for bit."""
    g, hq, hk, news = gen(7), 4, 2, [4, 1, 0]
    c = cu.Cache8(g, kind, 3, hk, d, 8, 3, layout)
    c.table[0, 2] = c.num_pages
    T, cu_new = sum(news), cumulated(news)
    cache, layers = c.describe(dtype, hq, 4, cu_new)
    rope = wkv.Rope(rot, 10000.0, order=order) if rot else None
    positions = torch.randint(0, 2 ** 20, (T,), generator=g).to(torch.int32).cuda()
    q, k, v = (randn(g, T, h, d, dtype=DT[dtype]) * (5.0 ** torch.randn((T, h, 1), generator=g)).to(DT[dtype]).cuda() for h in (hq, hk, hk))
    lengths = torch.tensor([[0, 14], [3, 23], [6, 22]], dtype=torch.int32, device="cuda")
    out, q_out = torch.full_like(lengths, 77), torch.full_like(q, 77.0)
    before = [x.clone() for x in c.codes[0] + c.scales[0]]
    wkv.wkv_append_kv_paged8(cache, layers[0], k, v, lengths, q=q, q_out=q_out, positions=positions, rope=rope, lengths_out=out)
    torch.cuda.synchronize()
    k_ref, q_ref = k.float().clone(), q.clone()
    if rot:
        wkv.wkv_norm_rotate_prompt(problem("f32", hq, hk, d, [T], "packed"), None, k_ref, None, k_ref, rope=rope, positions=positions)
        wkv.wkv_norm_rotate_prompt(problem(dtype, hq, hk, d, [T], "packed"), q_ref, None, q_ref, None, rope=rope, positions=positions)
        torch.cuda.synchronize()
    assert torch.equal(q_out, q_ref)
    for b, m in enumerate(news):
        for h in range(hk):
            n = int(lengths[b, h])
            assert int(out[b, h]) == min(n + m, c.cap)
            for kv, x in enumerate((k_ref, v)):
                scales, ref = cu.quantised(x[cu_new[b]:cu_new[b] + m, h], kind)
                codes, got_scales, ok = c.raw(0, kv, b, h, c.cap)
                for i in range(m):
                    if n + i < c.cap and ok[n + i]:
                        assert got_scales[n + i] == scales[i]
                        assert torch.equal(cu.values(codes[n + i], got_scales[n + i], kind), ref[i])
    # nothing else is written: of the rows with a page, those of the new tokens
    changed = [(x != y) for x, y in zip(c.codes[0] + c.scales[0], before)]
    for b, m in enumerate(news):
        for h in range(hk):
            for i in range(m):
                row = int(lengths[b, h]) + i
                if row >= c.cap or not 0 <= int(c.table[b, row // c.page]) < c.num_pages:
                    continue
                for kv in range(2):
                    pool_row(c, changed[kv], b, h, row)[:] = False
                    changed[2 + kv][int(c.table[b, row // c.page]), h, row % c.page] = False
    assert not any(bool(x.any()) for x in changed)


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_append8_with_norm(kind):
    """With norms and axes: what is read back is within the turned key's own error and half a step of a code (a scale that is a step larger included)."""
    g, hq, hk, d, T = gen(8), 4, 2, 128, 40
    case = ("bf16", d, True, 128, "half", 3, 1.0)
    c = cu.Cache8(g, kind, 1, hk, d, 16, 3)
    cache, layers = c.describe("bf16", hq, T)
    kw, weights, axis, positions = turn_setup(*case, T, g)
    k, v = randn(g, 1, hk, T, d, dtype=torch.bfloat16), randn(g, 1, hk, T, d, dtype=torch.bfloat16)
    lengths = torch.zeros((1, hk), dtype=torch.int32, device="cuda")
    wkv.wkv_append_kv_paged8(cache, layers[0], k, v, lengths, positions=positions.view(3, 1, T).cuda(), **kw)
    out = torch.full((1, hk, T, d), 77.0, device="cuda")
    wkv.wkv_read_kv_paged8(cache, layers[0], lengths + T, out, None)
    torch.cuda.synchronize()
    ref, big = cu.turned(k[0].transpose(0, 1), weights[1], 1e-5, 0.25, positions, axis, ou.frequencies(128, 500000.0), "half")
    own = cu.turned_bound(big, positions, d, 1.0, True)
    top = ref.abs().amax(-1, keepdim=True) + own
    step = ref.abs() * 2.0 ** -4 + 2 * top / 448 * 2.0 ** -10 if kind == "e4m3" else (2 * top / 127) / 2
    ou.assert_close(out[0].transpose(0, 1).cpu(), ref, own * (1 + 2.0 ** -4) + step * (1 + 2.0 ** -20), "key")


EDGES = [0.0, 1.0, -1.0, 448.0, 449.0, 447.9, 464.0, 127.0, 127.4, 127.5, 128.0, 1e-45, 2.0 ** -126, 2.0 ** -107, 1e-30, 3e38, -3e38, 2.0 ** 100, 127 * 2.0 ** 100,
         448 * 2.0 ** 100, 0.4375, 448 * 2.0 ** -100, 127 * 2.0 ** -100, INF, -INF, NAN]


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantised_rows_at_the_edges(kind, dtype):
    """Rows whose largest element is each of the edge values, beside fractions of it down to ties and below the least code."""
    d, rows = 64, []
    for top in EDGES:
        other = 3.0 if not np.isfinite(top) else top
        rows.append(torch.tensor([top] + [other * f for f in np.concatenate([np.arange(1, 33) / 33.0, 2.0 ** -np.arange(31.0)])], dtype=torch.float64).to(DT[dtype]))
    for most in (448, 127):          # halves between whole codes, and between the finest ones
        rows.append(torch.tensor([most] + [i / 2 for i in range(63)], dtype=torch.float64).to(DT[dtype]))
        rows.append(torch.tensor([-most] + [i * 2.0 ** -10 for i in range(63)], dtype=torch.float64).to(DT[dtype]))
    x = torch.stack(rows).cuda()                                          # [rows, d]
    n = len(rows)
    c = cu.Cache8(gen(1), kind, 1, 1, d, 16, (n + 15) // 16)
    cache, layers = c.describe(dtype, 1, n)
    kv = x.view(1, 1, n, d)
    wkv.wkv_append_kv_paged8(cache, layers[0], kv.flip(2).contiguous(), kv, torch.zeros((1, 1), dtype=torch.int32, device="cuda"))
    outs = {t: [torch.full((1, 1, n, d), 77.0, dtype=t, device="cuda") for _ in range(2)] for t in DT.values()}
    for t, (k_out, v_out) in outs.items():
        wkv.wkv_read_kv_paged8(cache, layers[0], torch.full((1, 1), n, dtype=torch.int32, device="cuda"), k_out, v_out)
    torch.cuda.synchronize()
    scales, ref = cu.quantised(x, kind)
    for i, (s, r) in enumerate(((scales.flip(0), ref.flip(0)), (scales, ref))):
        codes, got, _ = c.raw(0, i, 0, 0, n)
        assert torch.equal(got, s)
        assert torch.equal(torch.nan_to_num(cu.values(codes, got, kind), 9e99), torch.nan_to_num(r, 9e99))
        for t in DT.values():
            assert torch.equal(torch.nan_to_num(outs[t][i][0, 0].double(), 9e99), torch.nan_to_num(r, 9e99))          # exact in both types


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_read_every_code_and_scale(kind):
    """All 256 codes under every scale byte; fp32 holds them all (2^-127 times a code of 2^-9 is below its range and counts as what fp32 makes of it)."""
    c = cu.Cache8(gen(1), kind, 1, 1, 256, 16, 16)
    cache, layers = c.describe("f32", 1, 1)
    codes = torch.arange(256, dtype=torch.uint8).view(1, 256).expand(256, 256).cuda()
    for kv in range(2):
        c.put(0, kv, 0, 0, torch.arange(256), codes, torch.arange(256, dtype=torch.uint8).cuda())
    out = torch.full((1, 1, 256, 256), 77.0, device="cuda")
    wkv.wkv_read_kv_paged8(cache, layers[0], torch.full((1, 1), 256, dtype=torch.int32, device="cuda"), None, out)
    torch.cuda.synchronize()
    ref = cu.values(codes, torch.arange(256, dtype=torch.uint8).cuda(), kind).float()
    tiny = ref.abs() < 2.0 ** -126
    assert torch.equal(torch.nan_to_num(out[0, 0], 9e30)[~tiny], torch.nan_to_num(ref, 9e30)[~tiny]) and (out[0, 0][tiny].abs() <= 2.0 ** -126).all()


@pytest.mark.parametrize("layout", ["phsd", "pshd"])
def test_read_ranges(layout):
    g = gen(9)
    c = cu.Cache8(g, "i8", 2, 2, 48, 8, 20, layout)
    c.table[1, 1] = -1
    lengths = torch.tensor([[160, 33], [40, 0]], dtype=torch.int32, device="cuda")
    c.fill(g, lengths)
    cache, layers = c.describe("bf16", 4, 1)
    first = torch.tensor([[3, 40], [-2, 0]], dtype=torch.int32, device="cuda")
    for first_arg, capacity in ((None, 160), (first, 150), (first, 7)):
        out = [torch.full((2, 2, capacity, 48), 77.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        wkv.wkv_read_kv_paged8(cache, layers[0], lengths, out[0], out[1], first=first_arg)
        torch.cuda.synchronize()
        for kv in range(2):
            for b in range(2):
                for h in range(2):
                    want = torch.full((capacity, 48), 77.0, dtype=torch.float64, device="cuda")
                    n, f = int(lengths[b, h]), max(0, int(first[b, h])) if first_arg is not None else 0
                    ref, ok = c.rows(0, kv, b, h, n)
                    m = max(0, min(n - f, capacity))
                    want[:m][ok[f:f + m]] = ref[f:f + m][ok[f:f + m]]
                    assert torch.equal(out[kv][b, h].double(), want)


# ---- the gather behind the selection ----------------------------------------------------------------
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype,layout,pages,d,lens,alpha,omega,share", [
    ("bf16", "bhnd", "phsd", 64, [300, 300], 8, 8, 0.3), ("bf16", "packed", "pshd", 128, [1, 517, 33, 260], 16, 13, 0.5), ("f32", "bnhd", "phsd", 80, [400], 4, 32, 0.2),
    ("f32", "packed", "pshd", 256, [90, 7], 32, 4, 1.0), ("bf16", "packed", "phsd", 16, [2000], 1, 64, 0.9), ("bf16", "bhnd", "phsd", 64, [40], 64, 8, 0.5)])
def test_gather8(kind, dtype, layout, pages, d, lens, alpha, omega, share):
    """The rows of the selected windows and the observation rows, quantised; all others as they were."""
    g, hq, hk, B = gen(10), 4, 2, len(lens)
    kw = [max(0, (n - alpha + omega - 1) // omega) for n in lens]
    ks = [int(w * share) for w in kw]
    prob = problem(dtype, hq, hk, d, lens, layout, alpha, omega, [alpha + k * omega for k in ks])
    n, page = max(lens), 16
    max_pages = (prob.keep_max + page - 1) // page + 1
    idx = torch.full((B, hk, prob.k_max), -1, dtype=torch.int32)
    for b in range(B):
        for h in range(hk):
            some = torch.randperm(kw[b], generator=g)[: ks[b]].sort().values
            if h == 0 and ks[b] > 0:
                some[-1] = kw[b] - 1                                      # with the sequence's short last window
            idx[b, h, : ks[b]] = some.to(torch.int32)
    if ks[0] > 1:
        idx[0, 1, 0] = kw[0] + 3                                         # no window: its rows stay
    layers = 2
    shape = {"bhnd": (B, hk, n, d), "bnhd": (B, n, hk, d), "packed": (sum(lens), hk, d)}[layout]
    kx, vx = [[randn(g, *shape, dtype=DT[dtype]) for _ in range(layers)] for _ in range(2)]
    for t in kx + vx:
        t.view(-1, d)[7] *= 100
        t.view(-1, d)[-1, 0] = INF
    c = cu.Cache8(g, kind, B, hk, d, page, max_pages, pages, layers)
    if B > 1:
        c.table[0, 0] = -1
    cache, l8 = c.describe(dtype, hq)
    before = [x.clone() for l in range(layers) for x in c.codes[l] + c.scales[l]]
    wkv.wkv_gather_kv_paged8(prob, cache, l8, kx, vx, idx.cuda())
    torch.cuda.synchronize()
    for b, N in enumerate(lens):
        for h in range(hk):
            source = []
            for w in idx[b, h, : ks[b]].tolist():
                rows = list(range(w * omega, min((w + 1) * omega, N - alpha))) if w < kw[b] else [-1] * omega
                source += rows
            source += list(range(max(0, N - alpha), N))
            for l in range(layers):
                for kv, x in enumerate((kx[l], vx[l])):
                    mine = x[sum(lens[:b]):sum(lens[:b]) + N, h] if layout == "packed" else (x[b, h] if layout == "bhnd" else x[b, :, h])
                    at = torch.tensor(source, device="cuda")
                    scales, ref = cu.quantised(mine[at.clamp(min=0)], kind)
                    codes, got, ok = c.raw(l, kv, b, h, c.cap)
                    m = len(source)
                    live = ok[:m] & (at >= 0)
                    assert torch.equal(got[:m][live], scales[live])
                    assert torch.equal(torch.nan_to_num(cu.values(codes[:m], got[:m], kind)[live], 9e99), torch.nan_to_num(ref[live], 9e99))
                    assert (got[:m][~live & ok[:m]] == 255).all() and (codes[m:][ok[m:]] == 0x7f).all() and (got[m:][ok[m:]] == 255).all()
    used = torch.zeros(c.num_pages, dtype=torch.bool)
    t = c.table.cpu().flatten().long()
    used[t[(t >= 0) & (t < c.num_pages)]] = True
    for x, y in zip([x for l in range(layers) for x in c.codes[l] + c.scales[l]], before):
        assert torch.equal(x[~used.cuda()], y[~used.cuda()])


# ---- attention -------------------------------------------------------------------------------------
class Attend:
    """A cache, its description and a call's tensors, filled with what must not stay or must."""

    def __init__(self, dtype, kind, hq, hk, d, page, layout, lengths, news, packed, sees=None, seed=11, hole=None):
        g = gen(seed)
        self.dtype, self.kind, self.hq, self.hk, self.d, self.news, self.packed, self.sees = DT[dtype], kind, hq, hk, d, news, packed, sees
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        B = len(news)
        max_pages = (max(max(l) for l in lengths) + page - 1) // page + 1
        plain = kind == "plain"
        self.c = ou.Cache(g, self.dtype, B, hk, d, page, max_pages, layout) if plain else cu.Cache8(g, kind, B, hk, d, page, max_pages, layout)
        if hole is not None:
            self.c.table[hole] = -1
        self.c.fill(g, lengths)
        self.cu = cumulated(news)
        most = max(max(news), 1)
        cu_new = self.cu if packed else None
        if plain:
            self.cache = wkv.PagedCache(dtype=dtype, batch=B, n_q_heads=hq, n_kv_heads=hk, head_dim=d, page_size=page, num_pages=self.c.num_pages,
                                        block_table=self.c.table, max_new=most, cu_new=cu_new, layout=layout)
        else:
            self.cache, self.layers = self.c.describe(dtype, hq, most, cu_new)
        shape = (sum(news), hq, d) if packed else (B, hq, most, d)
        self.q = randn(g, *shape, dtype=self.dtype)
        self.out, self.lse = torch.full_like(self.q, 77.0), torch.full((B, hq, most), 77.0, device="cuda")
        self.ws = self.cache.alloc_workspace()
        self.weights = torch.rand((B, hk, self.c.cap), generator=g).cuda()
        self.weights_out = torch.full_like(self.weights, 77.0)
        self.masks = None
        if sees is not None:
            words = (most + 31) // 32
            masks = torch.full((B, most, words), -1, dtype=torch.int32)   # (bits behind a sequence's tokens do not count)
            for b, m in enumerate(news):
                w = cu.words_of(sees[b])
                masks[b, :m, : w.shape[1]] = w
                if m % 32:
                    masks[b, :m, m // 32] |= -1 << (m % 32)
            self.masks = (torch.cat([masks[b, :m] for b, m in enumerate(news)]) if packed else masks).contiguous().cuda()

    def run(self, weights=False, stream=None):
        if self.kind == "plain":
            wkv.wkv_attend_draft_paged(self.cache, self.masks, self.q, self.c.k[0], self.c.v[0], self.lengths, self.out, self.ws, lse=self.lse, stream=stream)
        else:
            more = dict(weights_in=self.weights, weights_out=self.weights_out) if weights else {}
            wkv.wkv_attend_paged8(self.cache, self.layers[0], self.q, self.lengths, self.out, self.ws, lse=self.lse, draft=self.masks, stream=stream, **more)

    def part(self, t, b, h):
        return t[self.cu[b]:self.cu[b + 1], h] if self.packed else t[b, h, : self.news[b]]

    def rows(self, kv, b, h, n):
        if self.kind == "plain":
            return self.c.rows((self.c.v if kv else self.c.k)[0], b, h, n)
        return self.c.rows(0, kv, b, h, n)

    def seen(self, b, h):
        n, m = int(self.lengths[b, h]), self.news[b]
        j, i = torch.arange(n)[None, :] - (n - m), torch.arange(m)[:, None]
        if self.sees is None:
            return (j <= i).cuda()
        return ((j < 0) | self.sees[b].gather(1, j.clamp(min=0).expand(m, n))).cuda() if m else torch.zeros((0, n), dtype=torch.bool).cuda()

    def check(self, weights=False):
        torch.cuda.synchronize()
        assert wkv.device_status(self.ws) == 0
        G = self.hq // self.hk
        for b, m in enumerate(self.news):
            for h in range(self.hk):
                n = int(self.lengths[b, h])
                (k, ok), (v, _) = self.rows(0, b, h, n), self.rows(1, b, h, n)
                seen = self.seen(b, h) & ok[None, :]
                received, slack = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
                for head in range(h * G, h * G + G):
                    ref, lse, p, bd = cu.attention_seen(self.part(self.q, b, head), k, v, seen)
                    ou.assert_close(self.part(self.out, b, head), ref, ou.output_bound(ref, bd, self.dtype), f"out {b} {head}")
                    ou.assert_close(self.lse[b, head, :m], lse, ou.lse_bound(lse, bd), f"lse {b} {head}")
                    assert (self.lse[b, head, m:] == 77.0).all()
                    received += p.sum(0)
                    slack += (bd["factor"][:, None] * p).sum(0)
                if weights:
                    ref = self.weights[b, h, :n].double() + received
                    bound = slack * 2 + (m * G + 4) * ou.U * ref
                    ou.assert_close(self.weights_out[b, h, :n], ref, bound, f"weights {b} {h}")
                    assert (self.weights_out[b, h, n:] == 77.0).all()


ATTEND = [
    # dtype, kind, hq, hk, d, page, layout, lengths, news, packed, hole
    ("bf16", "e4m3", 4, 1, 128, 16, "phsd", [[1]], [1], False, None),
    ("bf16", "i8", 8, 2, 128, 16, "phsd", [[992, 990]], [1], False, None),
    ("bf16", "e4m3", 8, 8, 64, 64, "pshd", [[70] * 8, [5] * 8], [1, 1], False, None),
    ("bf16", "i8", 6, 2, 80, 24, "phsd", [[333, 64], [65, 0]], [1, 1], True, (0, 1)),
    ("bf16", "e4m3", 16, 1, 96, 7, "pshd", [[500]], [1], False, (0, 2)),
    ("bf16", "i8", 12, 1, 128, 32, "phsd", [[260]], [1], False, None),
    ("bf16", "e4m3", 4, 2, 256, 16, "phsd", [[200, 31]], [2], False, None),
    ("bf16", "i8", 9, 1, 256, 16, "phsd", [[130]], [1], False, None),
    ("bf16", "i8", 4, 2, 16, 8, "phsd", [[40, 41], [3, 2]], [3, 2], True, None),
    ("bf16", "e4m3", 2, 1, 128, 16, "phsd", [[3000]], [4], False, None),
    ("bf16", "e4m3", 4, 2, 128, 64, "phsd", [[400, 397], [130, 128], [20, 21]], [5, 0, 20], True, None),
    ("bf16", "i8", 8, 2, 64, 16, "pshd", [[700, 699]], [70], False, (0, 3)),
    ("bf16", "e4m3", 32, 8, 128, 128, "phsd", [[1500] * 8], [130], False, None),
    ("bf16", "i8", 6, 1, 80, 8, "phsd", [[300], [90]], [90, 33], True, None),
    ("bf16", "e4m3", 4, 1, 256, 16, "phsd", [[150]], [40], False, None),
    ("bf16", "i8", 4, 1, 128, 6, "phsd", [[150]], [40], False, None),
    ("bf16", "i8", 2, 2, 112, 40, "pshd", [[2500, 2400]], [600], False, None),
    ("f32", "i8", 4, 2, 64, 24, "phsd", [[100, 99], [7, 7]], [7, 1], True, None),
    ("f32", "e4m3", 4, 2, 128, 16, "pshd", [[300, 10]], [1], False, (0, 0)),
    ("f32", "e4m3", 8, 1, 80, 16, "phsd", [[700]], [30], False, None),
    ("f32", "i8", 3, 3, 256, 16, "phsd", [[90, 80, 33]], [5], False, None),
    ("f32", "e4m3", 8, 2, 128, 16, "phsd", [[2600, 2001]], [1], False, (0, 5)),
    ("f32", "i8", 4, 1, 64, 24, "pshd", [[3001], [40]], [3, 1], True, None),
]


def name_of(c):
    return "-".join(map(str, c)).replace(" ", "").replace("(", "").replace(")", "")


@pytest.mark.parametrize("case", ATTEND, ids=name_of)
def test_attend8(case):
    a = Attend(*case[:10], hole=case[10])
    a.run()
    a.check()


@pytest.mark.parametrize("case", [ATTEND[i] for i in (0, 1, 2, 3, 4, 6, 8, 10, 12, 13, 14, 17, 18, 19, 21, 22)], ids=name_of)
def test_attend8_weights(case):
    a = Attend(*case[:10], hole=case[10])
    a.run(weights=True)
    a.check(weights=True)
    # in place, without any before
    b = Attend(*case[:10], hole=case[10])
    b.weights.zero_()
    b.weights_out = b.weights
    b.run(weights=True)
    torch.cuda.synchronize()
    for i in range(len(b.news)):
        for h in range(b.hk):
            n = int(b.lengths[i, h])
            got = (a.weights[i, h, :n] + b.weights[i, h, :n]).double()
            assert ((got - a.weights_out[i, h, :n]).abs() <= 4 * ou.U * got).all()


@pytest.mark.parametrize("dtype,d,G,new", [("bf16", 128, 4, 1), ("bf16", 64, 16, 1), ("bf16", 128, 4, 40), ("bf16", 256, 4, 10), ("f32", 64, 4, 6)])
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_attend8_does_not_see_what_is_hidden(dtype, d, G, new, kind):
    """NaN rows, by their scale or (E4M3) by a code, do not reach the queries in front of them, and reach those behind, however small their weight."""
    a = Attend(dtype, kind, G, 1, d, 16, "phsd", [[90]], [new], False)
    a.run()
    torch.cuda.synchronize()
    clean, clean_lse = a.out.clone(), a.lse.clone()
    at = 90 - new + new // 2                                              # the key of query new // 2
    codes, scales, _ = a.c.raw(0, 1, 0, 0, 90)
    scales[at] = 255
    a.c.put(0, 1, 0, 0, torch.arange(90), codes, scales)
    a.run()
    torch.cuda.synchronize()
    i = new // 2
    assert torch.equal(a.out[0, :, :i], clean[0, :, :i]) and torch.equal(a.lse, clean_lse)
    assert torch.isnan(a.out[0, :, i:]).all()
    if kind == "e4m3":
        scales[at] = 120
        codes[at, 5] = 0xff
        a.c.put(0, 1, 0, 0, torch.arange(90), codes, scales)
        a.run()
        torch.cuda.synchronize()
        assert torch.equal(a.out[0, :, :i], clean[0, :, :i])
        assert torch.isnan(a.out[0, :, i:, 5]).all() and torch.isfinite(a.out[0, :, i:, :5]).all() and torch.isfinite(a.out[0, :, i:, 6:]).all()
    codes, scales, _ = a.c.raw(0, 0, 0, 0, 90)
    scales[at] = 255
    a.c.put(0, 0, 0, 0, torch.arange(90), codes, scales)
    a.run()
    torch.cuda.synchronize()
    assert torch.equal(a.out[0, :, :i], clean[0, :, :i]) and torch.equal(a.lse[0, :, :i], clean_lse[0, :, :i])
    assert torch.isnan(a.out[0, :, i:]).all() and torch.isnan(a.lse[0, :, i:]).all()


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 30), ("f32", 2)])
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_attend8_rows_of_very_different_sizes(dtype, new, kind):
    """Scales from 2^-60 to 2^40 in values, a sink key whose value is next to nothing, queries of 2^30 and 2^-30: nothing is lost or overflows."""
    a = Attend(dtype, kind, 4, 1, 128, 16, "phsd", [[400]], [new], False)
    codes, scales, _ = a.c.raw(0, 1, 0, 0, 400)
    scales.copy_(torch.randint(67, 168, (400,), generator=gen(3)).to(torch.uint8))
    a.c.put(0, 1, 0, 0, torch.arange(400), codes, scales)
    a.run()
    a.check()
    # nearly all weight on a key without a value
    codes, scales, _ = a.c.raw(0, 1, 0, 0, 400)
    scales.fill_(121)
    codes[0] = 0
    scales[0] = 27
    a.c.put(0, 1, 0, 0, torch.arange(400), codes, scales)
    k_codes, k_scales, _ = a.c.raw(0, 0, 0, 0, 400)
    k_scales.fill_(112)
    k_codes[0] = 0x70 if kind == "e4m3" else 127
    k_scales[0] = 121
    a.c.put(0, 0, 0, 0, torch.arange(400), k_codes, k_scales)
    a.q.fill_(0.6)
    a.run()
    a.check()
    for by, scale in ((2.0 ** 30, 127 - 39), (2.0 ** -30, 127 + 21)):
        k_scales.fill_(scale)
        a.c.put(0, 0, 0, 0, torch.arange(400), k_codes, k_scales)
        a.q.copy_((randn(gen(4), *a.q.shape) * by).to(a.q.dtype))
        a.run()
        a.check()


# ---- drafts ----------------------------------------------------------------------------------------
def random_tree(g, m, roots=0.15):
    return [-1 if i == 0 or float(torch.rand((), generator=g)) < roots else int(torch.randint(0, i, (), generator=g)) for i in range(m)]


DRAFTS = [
    # dtype, kind, hq, hk, d, page, layout, lengths, news, packed, tree, hole
    ("bf16", "plain", 4, 1, 128, 16, "phsd", [[1]], [1], False, True, None),
    ("bf16", "plain", 4, 2, 128, 16, "phsd", [[992, 990]], [2], False, True, None),
    ("bf16", "plain", 8, 2, 64, 8, "pshd", [[70, 71], [12, 9], [5, 4]], [12, 9, 0], True, True, (0, 4)),
    ("bf16", "plain", 32, 8, 128, 64, "phsd", [[1300] * 8, [64] * 8], [64, 33], True, True, None),
    ("bf16", "plain", 3, 1, 80, 24, "phsd", [[700]], [150], False, False, None),
    ("bf16", "plain", 2, 1, 256, 16, "phsd", [[90]], [31], False, False, None),
    ("bf16", "plain", 4, 1, 128, 6, "phsd", [[300]], [20], False, True, None),
    ("bf16", "plain", 2, 2, 64, 32, "phsd", [[256, 258]], [256], False, False, None),
    ("bf16", "e4m3", 8, 2, 128, 16, "phsd", [[992, 990]], [2], False, True, None),
    ("bf16", "i8", 4, 1, 64, 16, "pshd", [[200], [40]], [4, 3], True, False, None),
    ("bf16", "e4m3", 32, 8, 128, 64, "pshd", [[1300] * 8, [64] * 8], [64, 33], True, True, (0, 3)),
    ("bf16", "i8", 4, 2, 96, 128, "phsd", [[1024, 1000]], [300], False, False, None),
    ("bf16", "e4m3", 4, 1, 256, 16, "phsd", [[70]], [17], False, True, None),
    ("f32", "plain", 4, 2, 64, 24, "phsd", [[500, 499], [9, 12]], [9, 5], True, True, None),
    ("f32", "plain", 2, 1, 128, 16, "phsd", [[160]], [100], False, False, None),
    ("f32", "i8", 4, 2, 80, 16, "pshd", [[150, 149]], [20], False, True, None),
    ("f32", "e4m3", 3, 1, 256, 16, "phsd", [[60]], [33], False, False, None),
]


@pytest.mark.parametrize("case", DRAFTS, ids=name_of)
def test_draft(case):
    """Trees, and masks of any form: later tokens, not the token itself, nothing at all."""
    g, news, tree = gen(13), case[8], case[10]
    sees = [cu.tree_of(random_tree(g, m)) if tree else torch.rand((m, m), generator=g) < 0.3 for m in news]
    if not tree:
        for s in sees:
            s[0] = False
    a = Attend(*case[:10], sees=sees, hole=case[11])
    a.run()
    a.check()


@pytest.mark.parametrize("dtype,kind,new", [("bf16", "plain", 12), ("bf16", "i8", 3), ("bf16", "e4m3", 40), ("f32", "plain", 12), ("bf16", "plain", 100)])
def test_draft_without_rows_in_front(dtype, kind, new):
    """Rows that see nothing give 0 and -infinity; a mask of all earlier tokens is the causal one."""
    sees = [torch.rand((new, new), generator=gen(2)) < 0.3]
    sees[0][new // 2] = False
    a = Attend(dtype, kind, 4, 2, 64, 16, "phsd", [[new, new]], [new], False, sees=sees)
    a.run()
    a.check()
    assert (a.out[0, :, new // 2] == 0).all() and (a.lse[0, :, new // 2] == -INF).all()
    b = Attend(dtype, kind, 4, 2, 64, 16, "phsd", [[new, new]], [new], False, sees=[torch.tril(torch.ones((new, new), dtype=torch.bool))])
    b.run()
    b.check()
    b.sees = None                                                         # (the reference of new tokens one after the other)
    b.check()


@pytest.mark.parametrize("dtype,kind,new,d", [("bf16", "plain", 3, 128), ("bf16", "plain", 40, 64), ("f32", "plain", 7, 64), ("bf16", "e4m3", 2, 128),
                                              ("bf16", "e4m3", 40, 128), ("bf16", "i8", 40, 64)])
def test_draft_does_not_see_other_branches(dtype, kind, new, d):
    """NaN (plain: infinities too) in the row of a token reaches its descendants and nobody else."""
    parents = random_tree(gen(5), new, 0.3)
    sees = cu.tree_of(parents)
    a = Attend(dtype, kind, 4, 1, d, 16, "phsd", [[100]], [new], False, sees=[sees])
    a.run()
    torch.cuda.synchronize()
    clean = a.out.clone()
    token = new // 3
    at = 100 - new + token
    if kind == "plain":
        a.c.slot(a.c.v[0], 0, 0, at)[3] = NAN
        a.c.slot(a.c.v[0], 0, 0, at)[5] = -INF
    else:
        codes, scales, _ = a.c.raw(0, 1, 0, 0, 100)
        if kind == "e4m3":
            codes[at, 3] = 0x7f
        else:
            scales[at] = 255
        a.c.put(0, 1, 0, 0, torch.arange(100), codes, scales)
    a.run()
    torch.cuda.synchronize()
    on = sees[:, token].cuda()
    assert torch.equal(a.out[0][:, ~on], clean[0][:, ~on])
    assert torch.isnan(a.out[0][:, on][..., 3]).all()
    if kind == "plain":
        assert (a.out[0][:, on][..., 5] == -INF).all()


@pytest.mark.parametrize("news,packed", [([1], False), ([40, 40], False), ([0, 33, 64, 1], True), ([1024], False)])
def test_draft_masks(news, packed):
    g, B, most = gen(14), len(news), max(news)
    table = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    cache = wkv.PagedCache(dtype="bf16", batch=B, n_q_heads=1, n_kv_heads=1, head_dim=8, page_size=16, num_pages=1, block_table=table, max_new=most,
                           cu_new=cumulated(news) if packed else None)
    parents = [random_tree(g, m) for m in news]
    if most > 8:
        parents[-1 if not packed else 1][7], parents[-1 if not packed else 1][5] = 7, 30          # itself, a later one: roots
    words = (most + 31) // 32 + 1
    shape = (sum(news),) if packed else (B, most)
    flat = torch.tensor([p for one in parents for p in one], dtype=torch.int32).view(shape).cuda()
    masks = torch.full(shape + (words,), 77, dtype=torch.int32, device="cuda")
    positions = torch.full(shape, 77, dtype=torch.int32, device="cuda")
    first = torch.randint(0, 1000, (B,), generator=g).to(torch.int32).cuda()
    wkv.wkv_draft_masks(cache, flat, masks, first, positions)
    torch.cuda.synchronize()
    off = 0
    for b, m in enumerate(news):
        sees = cu.tree_of(parents[b])
        part, pos = (masks[off:off + m], positions[off:off + m]) if packed else (masks[b], positions[b])
        off += m
        if m == 0:
            continue
        w = cu.words_of(sees)
        assert torch.equal(part[:, : w.shape[1]].cpu(), w) and (part[:, w.shape[1]:] == 0).all()
        assert torch.equal(pos.cpu(), (int(first[b]) + sees.sum(1) - 1).to(torch.int32))
    wkv.wkv_draft_masks(cache, flat, None, None, positions)
    torch.cuda.synchronize()
    assert int(positions.view(-1)[0]) == 0


@pytest.mark.parametrize("kind", ["plain", "f32", "e4m3"])
@pytest.mark.parametrize("layout", ["phsd", "pshd"])
def test_keep_draft(kind, layout):
    """The path's rows move down, rows without a page stay, lengths and the rows' state follow; everything else is as it was."""
    g, news, hk, d, page, layers = gen(15), [40, 1, 17, 0, 9], 2, 64, 8, 2
    lengths = [[90, 88], [5, 6], [17, 20], [7, 0], [30, 4]]               # (the last: a unit with fewer rows than the draft has tokens)
    B, cu_new = len(news), cumulated(news)
    parents = [random_tree(g, m, 0.05) for m in news]
    sees = [cu.tree_of(p) for p in parents]
    last = [39, 0, 17, 0, 8]                                              # (17: no token of its sequence)
    eight = kind == "e4m3"
    if eight:
        c = cu.Cache8(g, kind, B, hk, d, page, 12, layout, layers)
    else:
        c = ou.Cache(g, torch.float32 if kind == "f32" else torch.bfloat16, B, hk, d, page, 12, layout, layers, fill=55.0)
    c.table[0, 9] = -1
    c.fill(g, lengths)
    dtype = "f32" if kind == "f32" else "bf16"
    if eight:
        cache, l8 = c.describe(dtype, 2, 40, cu_new)
        tensors = [x for l in range(layers) for x in c.codes[l] + c.scales[l]]
    else:
        cache = wkv.PagedCache(dtype=dtype, batch=B, n_q_heads=2, n_kv_heads=hk, head_dim=d, page_size=page, num_pages=c.num_pages, block_table=c.table,
                               max_new=40, cu_new=cu_new, layout=layout)
        tensors = c.k + c.v
    masks = torch.zeros((sum(news), 2), dtype=torch.int32)
    for b, m in enumerate(news):
        w = cu.words_of(sees[b]) if m else torch.zeros((0, 1), dtype=torch.int32)
        masks[cu_new[b]:cu_new[b + 1], : w.shape[1]] = w
    before = [t.clone() for t in tensors]
    want = [t.clone() for t in tensors]
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    positions = torch.randint(0, 9999, (B, hk, c.cap), generator=g).to(torch.int32).cuda()
    weights = torch.rand((B, hk, c.cap), generator=g).cuda()
    want_pos, want_w, out, want_out = positions.clone(), weights.clone(), torch.full_like(lens, 77), lens.clone()
    for b, m in enumerate(news):
        path = [j for j in range(m) if 0 <= last[b] < m and sees[b][last[b], j]]
        for h in range(hk):
            n = lengths[b][h]
            rows = [n - m + j for j in path if n - m + j >= 0]
            to0 = max(n - m, 0)
            want_out[b, h] = to0 + len(rows)
            for x, r in enumerate(rows):
                want_pos[b, h, to0 + x], want_w[b, h, to0 + x] = positions[b, h, r], weights[b, h, r]
                src, dst = int(c.table[b, r // page]), int(c.table[b, (to0 + x) // page])
                if src < 0 or dst < 0:
                    continue
                for t, w in zip(before, want):
                    if t.dim() == 3 or layout == "phsd":
                        w[dst, h, (to0 + x) % page] = t[src, h, r % page]
                    else:
                        w[dst, (to0 + x) % page, h] = t[src, r % page, h]
    args = (torch.tensor(last, dtype=torch.int32, device="cuda"), lens, out, positions, weights)
    if eight:
        wkv.wkv_keep_draft_paged8(cache, masks.cuda(), l8, *args)
    else:
        wkv.wkv_keep_draft_paged(cache, masks.cuda(), c.k, c.v, *args)
    torch.cuda.synchronize()
    assert torch.equal(out, want_out) and torch.equal(positions, want_pos) and torch.equal(weights, want_w)
    for t, w in zip(tensors, want):
        assert torch.equal(torch.nan_to_num(t.float(), 9e30), torch.nan_to_num(w.float(), 9e30))


# ---- eviction --------------------------------------------------------------------------------------
@pytest.mark.parametrize("budget,cap_pages", [(20, 6), (200, 40), (300, 60), (0, 3), (1000, 6), (2, 6)])
@pytest.mark.parametrize("layout", ["phsd", "pshd"])
def test_evict8(budget, cap_pages, layout):
    """The rows' state as from the plain cache's eviction; codes and scales of every layer belong to the positions that stay."""
    g, B, hk, d, page, layers = gen(16), 3, 2, 48, 16, 3
    c = cu.Cache8(g, "e4m3", B, hk, d, page, cap_pages, layout, layers)
    cap = c.cap
    lens = torch.tensor([[cap, cap - 5], [cap // 2, 0], [33, 7]], dtype=torch.int32, device="cuda")
    lens.clamp_(max=cap)
    c.fill(g, lens.tolist())
    cache, l8 = c.describe("bf16", 2)
    plain = ou.Cache(g, torch.bfloat16, B, hk, 8, page, cap_pages, layout)
    pc = wkv.PagedCache(dtype="bf16", batch=B, n_q_heads=2, n_kv_heads=hk, head_dim=8, page_size=page, num_pages=c.num_pages, block_table=c.table, layout=layout)
    weights = torch.rand((B, hk, cap), generator=g).cuda()
    weights[:, :, ::7] = 0.5
    positions = torch.stack([torch.randperm(cap, generator=g) for _ in range(B * hk)]).view(B, hk, cap).to(torch.int32).cuda()
    held = {(l, kv, b, h): c.raw(l, kv, b, h, int(lens[b, h])) for l in range(layers) for kv in range(2) for b in range(B) for h in range(hk)}
    outs = [[torch.full_like(x, 77) for x in (weights, positions, lens)] for _ in range(2)]
    wkv.wkv_evict_kv_paged8(cache, l8, weights, positions, lens, budget, 3, *outs[0], cache.alloc_workspace())
    wkv.wkv_evict_kv_paged(pc, plain.k, plain.v, weights, positions, lens, budget, 3, *outs[1], pc.alloc_workspace())
    torch.cuda.synchronize()
    for x, y in zip(*outs):
        assert torch.equal(x, y)
    for (l, kv, b, h), (codes, scales, _) in held.items():
        n, keep = int(lens[b, h]), int(outs[0][2][b, h])
        row_of = {int(p): r for r, p in enumerate(positions[b, h, :n])}
        rows = torch.tensor([row_of[int(p)] for p in outs[0][1][b, h, :keep]], dtype=torch.long, device="cuda")
        now, now_scales, _ = c.raw(l, kv, b, h, keep)
        assert torch.equal(now, codes[rows]) and torch.equal(now_scales, scales[rows])


# ---- far places ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind,new", [("e4m3", 1), ("i8", 30), ("e4m3", 150)])
def test_offsets_beyond_32_bits(kind, new):
    """Pages a gigabyte apart: appended to, read back, attended over, kept of a draft."""
    g, hk, hq, d, page, gap = gen(18), 2, 8, 64, 16, 1 << 30
    n, num_pages, max_pages = 100, 12, 12
    if new == 150:
        n, num_pages, max_pages = 170, 12, 12
    codes = [torch.empty(gap * (num_pages - 1) + hk * page * d, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((num_pages, hk, page), dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device="cuda").view(1, max_pages)
    make = lambda m: wkv.PagedCache8(kind=kind, dtype="bf16", batch=1, n_q_heads=hq, n_kv_heads=hk, head_dim=d, page_size=page, num_pages=num_pages,
                                     block_table=table, max_new=m, layout=(gap, page * d, d))
    filling, cache = make(n), make(new)
    layer = wkv.Layer8(cache, *codes, *scales)
    k, v = (randn(g, 1, hk, n, d, dtype=torch.bfloat16) for _ in range(2))
    none, lengths = torch.zeros((1, hk), dtype=torch.int32, device="cuda"), torch.full((1, hk), n, dtype=torch.int32, device="cuda")
    wkv.wkv_append_kv_paged8(filling, layer, k, v, none)
    rows = [torch.full((1, hk, n, d), 77.0, device="cuda") for _ in range(2)]
    wkv.wkv_read_kv_paged8(filling, layer, lengths, rows[0], rows[1])
    q = randn(g, 1, hq, new, d, dtype=torch.bfloat16)
    out, ws = torch.full_like(q, 77.0), cache.alloc_workspace()
    wkv.wkv_attend_paged8(cache, layer, q, lengths, out, ws)
    torch.cuda.synchronize()
    seen = (torch.arange(n)[None, :] <= torch.arange(new)[:, None] + n - new).cuda()
    for h in range(hk):
        for x, y in ((k, rows[0]), (v, rows[1])):
            assert torch.equal(y[0, h].double(), cu.quantised(x[0, h], kind)[1])
        for head in range(h * 4, h * 4 + 4):
            ref, _, _, bd = cu.attention_seen(q[0, head], rows[0][0, h], rows[1][0, h], seen)
            ou.assert_close(out[0, head], ref, ou.output_bound(ref, bd, torch.bfloat16), "out")
    assert wkv.device_status(ws) == 0
    masks = torch.zeros((1, new, (new + 31) // 32), dtype=torch.int32, device="cuda")
    masks[0, -1, -1] = 1 << ((new - 1) % 32) if new % 32 else -2 ** 31     # the last token alone
    kept = torch.zeros_like(lengths)
    wkv.wkv_keep_draft_paged8(cache, masks, [layer], torch.tensor([new - 1], dtype=torch.int32, device="cuda"), lengths, kept)
    last = torch.full((1, hk, 1, d), 77.0, device="cuda")
    wkv.wkv_read_kv_paged8(filling, layer, kept, last, None, first=kept - 1)
    torch.cuda.synchronize()
    assert (kept == n - new + 1).all() and torch.equal(last[:, :, 0], rows[0][:, :, n - 1])


# ---- a run of them together ----------------------------------------------------------------------------
@pytest.mark.parametrize("kind,dtype", [("e4m3", "bf16"), ("i8", "bf16"), ("i8", "f32")])
def test_selection_to_drafts(kind, dtype):
    """A prompt's norms and rotation, its selection into an 8-bit cache, a few tokens with weights, the eviction, a draft and what is kept of it,
    and the next token; what attends is held to 64 bits over what the cache stands for at that time."""
    g, hq, hk, d, n, alpha, omega, page = gen(17), 8, 2, 64, 600, 8, 8, 16
    budget = 200
    prob = problem(dtype, hq, hk, d, [n], "bhnd", alpha, omega, [budget])
    rope, norm = wkv.Rope(d, 10000.0), wkv.HeadNorm((1 + 0.2 * torch.randn(d, generator=g)).to(DT[dtype]).cuda(), None, eps=1e-6)
    q, k, v = (randn(g, 1, h, n, d, dtype=DT[dtype]) for h in (hq, hk, hk))
    wkv.wkv_norm_rotate_prompt(prob, q, k, q, k, norm=norm, rope=rope)
    q_obs = q[:, :, n - alpha:].contiguous()
    ws = prob.alloc_workspace()
    scores, idx, kept = (torch.zeros(s, dtype=t, device="cuda") for s, t in (((1, hk, prob.kw_max), torch.float32), ((1, hk, prob.k_max), torch.int32), ((1, hk), torch.int32)))
    wkv.wkv_select_leader_windows(prob, q_obs, k, scores, idx, kept, ws)
    c = cu.Cache8(g, kind, 1, hk, d, page, 20)
    cache, (layer,) = c.describe(dtype, hq, 1)
    wkv.wkv_gather_kv_paged8(prob, cache, [layer], [k], [v], idx)
    positions = torch.zeros((1, hk, c.cap), dtype=torch.int32, device="cuda")
    weights = torch.zeros((1, hk, c.cap), device="cuda")
    wkv.wkv_seed_rows(prob, idx, None, positions, weights)
    lengths, space = kept.clone(), cache.alloc_workspace()

    def step(cache, space, m, at, parents=None):
        nonlocal lengths
        x = [randn(g, 1, h, m, d, dtype=DT[dtype]) for h in (hq, hk, hk)]
        masks, pos = None, torch.arange(at, at + m, dtype=torch.int32, device="cuda").view(1, m)
        if parents is not None:
            masks = torch.zeros((1, m, (m + 31) // 32), dtype=torch.int32, device="cuda")
            wkv.wkv_draft_masks(cache, torch.tensor([parents], dtype=torch.int32, device="cuda"), masks, torch.tensor([at], dtype=torch.int32, device="cuda"), pos)
        grown = torch.empty_like(lengths)
        wkv.wkv_append_kv_paged8(cache, layer, x[1], x[2], lengths, q=x[0], q_out=x[0], positions=pos, norm=norm, rope=rope, lengths_out=grown,
                                 row_positions=positions, row_weights=weights)
        out, lse = torch.full_like(x[0], 77.0), torch.full((1, hq, m), 77.0, device="cuda")
        more = dict(draft=masks) if parents is not None else dict(weights_in=weights, weights_out=weights)
        old = weights.clone()
        wkv.wkv_attend_paged8(cache, layer, x[0], grown, out, space, lse=lse, **more)
        torch.cuda.synchronize()
        for h in range(hk):
            N = int(grown[0, h])
            (kk, _), (vv, _) = c.rows(0, 0, 0, h, N), c.rows(0, 1, 0, h, N)
            j, i = torch.arange(N)[None, :] - (N - m), torch.arange(m)[:, None]
            seen = j <= i if parents is None else (j < 0) | cu.tree_of(parents).gather(1, j.clamp(min=0).expand(m, N))
            got, slack = (torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(2))
            for head in range(h * 4, h * 4 + 4):
                ref, ref_lse, p, bd = cu.attention_seen(x[0][0, head], kk, vv, seen.cuda())
                ou.assert_close(out[0, head], ref, ou.output_bound(ref, bd, DT[dtype]), "out")
                ou.assert_close(lse[0, head], ref_lse, ou.lse_bound(ref_lse, bd), "lse")
                got += p.sum(0)
                slack += (bd["factor"][:, None] * p).sum(0)
            if parents is None:
                ref = old[0, h, :N].double() + got
                ou.assert_close(weights[0, h, :N], ref, 2 * slack + (4 * m + 4) * ou.U * ref, "weights")
        lengths = grown
        return masks

    for t in range(5):
        step(cache, space, 1, n + t)
    out = torch.empty_like(lengths)
    wkv.wkv_evict_kv_paged8(cache, [layer], weights, positions, lengths, 150, 16, weights, positions, out, space)
    lengths = out
    assert (lengths == 150).all()
    m = 11
    drafting, _ = c.describe(dtype, hq, m)
    masks = step(drafting, drafting.alloc_workspace(), m, n + 5, [-1, 0, 0, 1, 1, 2, 3, 6, -1, 8, 7])
    kept_len = torch.empty_like(lengths)
    wkv.wkv_keep_draft_paged8(drafting, masks, [layer], torch.tensor([10], dtype=torch.int32, device="cuda"), lengths, kept_len, positions, weights)
    torch.cuda.synchronize()
    assert (kept_len == 156).all()                                        # tokens 0, 1, 3, 6, 7, 10
    assert positions[0, :, 150:156].tolist() == [list(range(n + 5, n + 11))] * hk
    lengths = kept_len
    step(cache, space, 1, n + 11)
    assert wkv.device_status(space) == 0


# ---- streams and graphs --------------------------------------------------------------------------------
@pytest.mark.parametrize("kind,new,draft", [("e4m3", 1, False), ("i8", 60, False), ("e4m3", 60, True), ("plain", 30, True), ("plain", 3, True)])
def test_calls_on_several_streams_and_captured(kind, new, draft):
    """Two calls at once on streams of their own, and a captured call replayed on other inputs, give what each gives alone."""
    def make(seed):
        sees = [cu.tree_of(random_tree(gen(seed), new)) for _ in range(2)] if draft else None
        return Attend("bf16", kind, 8, 2, 128, 16, "phsd", [[700, 690], [300, 299]], [new, new], False, sees=sees, seed=seed)
    a, b = make(1), make(2)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                x.run()
    a.check()
    b.check()
    torch.cuda.synchronize()
    want = b.out.clone()
    a.out.fill_(77.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    tensors = [(a.q, b.q)] + ([(a.masks, b.masks)] if draft else [])
    tensors += [(x, y) for x, y in zip(a.c.k + a.c.v, b.c.k + b.c.v)] if kind == "plain" else [(x, y) for x, y in zip(a.c.codes[0] + a.c.scales[0], b.c.codes[0] + b.c.scales[0])]
    for x, y in tensors + [(a.c.table, b.c.table)]:
        x.copy_(y)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.out, want)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.out, want)
    del graph
