"""CPU-only checks of the entry points around the selection: struct mirrors, the frequency table, refusals before any device work."""
import ctypes
import math

import numpy as np
import pytest

import operators_util as ou
from paper_2503_17922_b200 import binding, build


@pytest.fixture(scope="module")
def L():
    build.build_library()
    lib = binding.lib()
    lib.launched_before = lib.wkv_launch_count()
    return lib


P = 0x1000      # an aligned address that nothing follows: every call here is refused on the host


def shape(**kw):
    s = binding.WkvShape()
    s.struct_size = ctypes.sizeof(binding.WkvShape)
    s.dtype, s.batch, s.n_q_heads, s.n_kv_heads, s.head_dim = binding.WKV_BF16, 1, 4, 2, 64
    s.l_obs, s.window, s.top_p, s.task, s.max_seqlen, s.budget = 8, 8, 0, 0, 1024, 128
    s.stride_b, s.stride_h, s.stride_t = 2 * 1024 * 64, 1024 * 64, 64
    s.q_stride_b, s.q_stride_h, s.q_stride_t = 4 * 8 * 64, 8 * 64, 64
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def paged(**kw):
    c = binding.WkvPaged()
    c.struct_size = ctypes.sizeof(binding.WkvPaged)
    c.dtype, c.batch, c.n_q_heads, c.n_kv_heads, c.head_dim = binding.WKV_BF16, 2, 4, 2, 64
    c.max_new, c.page_size, c.num_pages, c.max_pages = 3, 16, 20, 8
    c.block_table = P
    c.page_stride, c.head_stride, c.row_stride = 2 * 16 * 64, 16 * 64, 64
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rope(**kw):
    r = binding.WkvRope(ctypes.sizeof(binding.WkvRope), 64, 0, 1.0, P)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def strides(*st):
    return (ctypes.c_int64 * 3)(*st)


QS = strides(4 * 1024 * 64, 1024 * 64, 64)
BIG = 1 << 40


def test_struct_mirrors():
    assert ctypes.sizeof(binding.WkvPaged) == 12 * 4 + 3 * 8 + 3 * 8
    assert ctypes.sizeof(binding.WkvRope) == 4 * 4 + 8


@pytest.mark.parametrize("rot,base,scaling,factor,original", [
    (128, 10000.0, "none", 1.0, 0.0), (64, 500000.0, "linear", 8.0, 0.0), (128, 500000.0, "base", 4.0, 0.0),
    (2, 10000.0, "base", 4.0, 0.0), (128, 500000.0, "bands", 8.0, 8192.0), (80, 10000.0, "bands", 32.0, 4096.0),
])
def test_frequencies_in_turns(L, rot, base, scaling, factor, original):
    got = binding.wkv_rope_frequencies(rot, base, scaling, factor, original)
    ref = ou.frequencies(rot, base, scaling, factor, original)
    # the reference is in 64 bits: relative 2^-50 of rounding errors, and half a unit of 2^-64 turns
    for g, f in zip(got, ref):
        assert abs(int(g) * 2.0 ** -64 - f / (2 * math.pi)) <= f * 2.0 ** -48 + 2.0 ** -64


def test_frequencies_wrap_whole_turns(L):
    got = binding.wkv_rope_frequencies(2, 1.0, "linear", 1.0 / (2 * math.pi * 3.25))
    assert abs(int(got[0]) * 2.0 ** -64 - 0.25) < 1e-12


@pytest.mark.parametrize("args", [
    (3, 1e4, "none", 1.0), (0, 1e4, "none", 1.0), (64, 0.0, "none", 1.0), (64, -1.0, "none", 1.0), (64, 1e4, "linear", 0.0),
    (64, 1e4, "bands", 2.0, 0.0), (64, 1e4, "bands", 2.0, 8192.0, 4.0, 4.0), (64, float("nan"), "none", 1.0), (64, 1e4, "linear", float("inf")),
])
def test_frequency_refusals(L, args):
    with pytest.raises(binding.WkvError) as e:
        binding.wkv_rope_frequencies(*args)
    assert e.value.status == 2


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), 2), (dict(dtype=5), 3), (dict(batch=0), 2), (dict(n_q_heads=3), 2), (dict(head_dim=4), 6),
    (dict(max_new=0), 2), (dict(page_size=0), 2), (dict(num_pages=0), 2), (dict(max_pages=0), 2), (dict(block_table=None), 1),
    (dict(row_stride=60), 6), (dict(row_stride=56), 2), (dict(page_stride=-64), 6), (dict(cu_new_host=P), 1), (dict(cu_new_dev=P), 1),
    (dict(max_pages=1 << 27), 9), (dict(page_size=1 << 30, max_pages=2), 9),
])
def test_paged_description_refusals(L, kw, status):
    c = paged(**kw)
    assert L.wkv_paged_workspace_bytes(ctypes.byref(c)) == 0
    ptrs = (ctypes.c_void_p * 2)(P, 2 * P)
    st = strides(4 * 3 * 64, 3 * 64, 64)
    calls = [
        L.wkv_append_kv_paged(ctypes.byref(c), None, P, P, st, None, None, None, P, P, P, 2 * P, None, None, None, None),
        L.wkv_attend_paged(ctypes.byref(c), P, st, P, P, P, 2 * P, st, None, None, None, P, BIG, None),
        L.wkv_evict_kv_paged(ctypes.byref(c), 2, ptrs, None, 1, None, 0, P, P, P, P, P, P, P, BIG, None),
    ]
    assert calls == [status] * 3, L.wkv_last_error_detail()
    assert L.wkv_last_error_detail()


def test_reserved_words(L):
    c = paged()
    c.reserved[1] = 1
    assert L.wkv_paged_workspace_bytes(ctypes.byref(c)) == 0
    assert L.wkv_paged_workspace_bytes(ctypes.byref(paged())) > 0
    assert L.wkv_paged_workspace_bytes(None) == 0


@pytest.mark.parametrize("cu", [[0, 4, 5], [1, 2, 3], [0, 2, 1]])
def test_chunk_lengths(L, cu):
    a = np.array(cu, dtype=np.int32)
    c = paged(cu_new_host=a.ctypes.data, cu_new_dev=P)
    assert L.wkv_paged_workspace_bytes(ctypes.byref(c)) == 0
    a[:] = [0, 0, 3]
    assert L.wkv_paged_workspace_bytes(ctypes.byref(c)) > 0


def test_attend_paged_refusals(L):
    c = paged()
    need = L.wkv_paged_workspace_bytes(ctypes.byref(c))
    st = strides(4 * 3 * 64, 3 * 64, 64)

    def call(q=P, qs=st, k=P, v=P, n=P, out=2 * P, os=st, lse=None, win=None, wout=None, ws=P, size=need, desc=c):
        return L.wkv_attend_paged(ctypes.byref(desc), q, qs, k, v, n, out, os, lse, win, wout, ws, size, None)

    assert [call(q=None), call(k=None), call(v=None), call(n=None), call(out=None), call(qs=None), call(os=None)] == [1] * 7
    assert [call(q=P + 8), call(k=P + 8), call(out=P + 8), call(qs=strides(64, 4, 64))] == [6] * 4
    assert [call(ws=None), call(size=need - 1), call(ws=P + 16)] == [5] * 3
    assert call(win=P) == 1 and call(out=P) == 2 and call(qs=strides(64, 64, 56)) == 2
    assert call(desc=paged(head_dim=264, page_stride=2 * 16 * 264, head_stride=16 * 264, row_stride=264), qs=strides(0, 264, 264), os=strides(0, 264, 264)) == 7


def test_append_refusals(L):
    c = paged()
    st = strides(2 * 3 * 64, 3 * 64, 64)

    def call(r=None, k=P, v=P, ks=st, q=None, qo=None, qs=None, pos=P, n=P, kp=P, vp=2 * P, no=None, rp=None, rw=None):
        return L.wkv_append_kv_paged(ctypes.byref(c), ctypes.byref(r) if r is not None else None, k, v, ks, q, qo, qs, pos, n, kp, vp, no, rp,
                                     rw, None)

    assert [call(k=None), call(v=None), call(ks=None), call(n=None), call(kp=None), call(vp=None), call(q=P), call(qo=P)] == [1] * 8
    assert [call(pos=None, r=rope()), call(pos=None, rp=P), call(q=P, qo=P, qs=None), call(r=rope(turns=None))] == [1] * 4
    assert [call(k=P + 8), call(kp=P + 8), call(ks=strides(0, 4, 64))] == [6] * 3
    assert [call(no=P), call(vp=P), call(ks=strides(0, 64, 32))] == [2] * 3
    assert [call(r=rope(struct_size=1)), call(r=rope(rot_dim=3)), call(r=rope(rot_dim=66)), call(r=rope(rot_dim=0)), call(r=rope(order=2)),
            call(r=rope(scale=math.inf)), call(r=rope(scale=math.nan))] == [2] * 7


def test_evict_refusals(L):
    c = paged()
    need = L.wkv_paged_workspace_bytes(ctypes.byref(c))
    ptrs = (ctypes.c_void_p * 40)(*([P] * 40))

    def call(layers=1, k=ptrs, v=None, budget=4, recent=0, w=P, p=P, n=P, wo=P, po=P, no=P, ws=P, size=need):
        return L.wkv_evict_kv_paged(ctypes.byref(c), layers, k, v, budget, None, recent, w, p, n, wo, po, no, ws, size, None)

    assert [call(layers=0), call(layers=33)] == [9] * 2
    assert [call(k=None), call(w=None), call(p=None), call(n=None), call(wo=None), call(po=None), call(no=None)] == [1] * 7
    assert call(budget=-1) == 4 and call(recent=-1) == 2
    assert [call(ws=None), call(size=need - 1), call(ws=P + 128)] == [5] * 3
    assert call(k=(ctypes.c_void_p * 1)(P + 8)) == 6 and call(k=(ctypes.c_void_p * 1)(None)) == 1


def test_prompt_refusals(L):
    def attend(s=None, q=P, qs=QS, k=P, v=P, out=2 * P, os=QS):
        return L.wkv_attend_prompt(ctypes.byref(s if s is not None else shape()), q, qs, k, v, out, os, None, None, None, None)

    assert [attend(q=None), attend(k=None), attend(v=None), attend(out=None), attend(qs=None), attend(os=None)] == [1] * 6
    assert [attend(q=P + 4), attend(v=P + 8), attend(qs=strides(0, 4, 64)), attend(qs=strides(-64, 64, 64))] == [6] * 4
    assert [attend(out=P), attend(qs=strides(0, 64, 32)), attend(s=shape(batch=0))] == [2] * 3
    assert attend(s=shape(head_dim=264, stride_t=264, q_stride_t=264), qs=strides(0, 264, 264), os=strides(0, 264, 264)) == 7

    def rotate(r=None, q=P, qo=P, qs=QS, k=P, ko=P, s=None):
        return L.wkv_rotate_prompt(ctypes.byref(s if s is not None else shape()), ctypes.byref(r if r is not None else rope()), q, qo, qs, k, ko,
                                   None, None)

    assert [rotate(q=None), rotate(ko=None), rotate(qs=None), rotate(q=None, qo=None, k=None, ko=None), rotate(r=rope(turns=None))] == [1] * 5
    assert [rotate(q=P + 8), rotate(k=P + 8)] == [6] * 2
    assert [rotate(r=rope(rot_dim=66)), rotate(r=rope(order=-1)), rotate(qs=strides(0, 64, 8))] == [2] * 3
    assert L.wkv_rotate_prompt(ctypes.byref(shape()), None, P, P, QS, P, P, None, None) == 1


def test_seed_refusals(L):
    s = shape()
    assert L.wkv_keep_max(ctypes.byref(s)) == 128
    assert L.wkv_seed_rows(ctypes.byref(s), None, None, 128, P, P, None) == 1
    assert L.wkv_seed_rows(ctypes.byref(s), P, None, 128, None, None, None) == 1
    assert L.wkv_seed_rows(ctypes.byref(s), P, None, 127, P, P, None) == 2


def test_nothing_was_launched(L):
    assert L.wkv_launch_count() == L.launched_before


def test_python_side_checks_shapes():
    torch = pytest.importorskip("torch")
    t = torch.zeros((2, 4, 3, 64), dtype=torch.bfloat16)
    assert list(binding._head_strides(t, False, "q")) == [768, 192, 64]
    assert list(binding._head_strides(t[0].transpose(0, 1), True, "q")) == [0, 192, 64]
    with pytest.raises(ValueError):
        binding._head_strides(t[0], False, "q")
    with pytest.raises(ValueError):
        binding._head_strides(t.transpose(2, 3), False, "q")
    with pytest.raises(ValueError):
        binding._check_heads(t, 4, torch.float32, 64, False, 2, 3, "q")
    with pytest.raises(ValueError):
        binding._check_heads(t, 4, torch.bfloat16, 64, False, 2, 4, "q")
    with pytest.raises(ValueError):
        binding._check_state(torch.zeros((2, 2), dtype=torch.int64), (2, 2), "int32", "lengths")
    with pytest.raises(ValueError):
        binding._check_state(torch.zeros((2, 4), dtype=torch.int32)[:, ::2], (2, 2), "int32", "lengths")
    with pytest.raises(ValueError):
        binding._check_same_layout(t, t.transpose(1, 2), "q and q_out")


def test_binding_refuses_pools_and_keys_that_are_too_small():
    import torch
    table = torch.zeros((2, 4), dtype=torch.int32)
    cache = binding.PagedCache(dtype="bf16", batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, num_pages=6, block_table=table)
    q, n, ws = torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16), torch.zeros((2, 2), dtype=torch.int32), torch.zeros(8, dtype=torch.uint8)
    pool = torch.zeros((6, 2, 16, 64), dtype=torch.bfloat16)
    for bad in (pool[:5].clone(), pool.float(), pool.view(-1)[64:]):
        with pytest.raises(ValueError, match="pool"):
            binding.prepare_attend_paged(cache, q, bad, pool, n, q.clone(), ws)
        with pytest.raises(ValueError, match="pool"):
            binding.prepare_attend_paged(cache, q, pool, bad, n, q.clone(), ws)
        with pytest.raises(ValueError, match="pool"):
            binding.prepare_append_kv_paged(cache, q[:, :2], q[:, :2], n, bad, pool)
        w, pos = torch.zeros((2, 2, 64)), torch.zeros((2, 2, 64), dtype=torch.int32)
        with pytest.raises(ValueError, match="pool"):
            binding.prepare_evict_kv_paged(cache, [pool, bad], None, w, pos, n, 8, 2, w, pos, n, ws)
    with pytest.raises(ValueError, match="per layer"):
        binding.prepare_evict_kv_paged(cache, [pool, pool], [pool], w, pos, n, 8, 2, w, pos, n, ws)


def problem(**kw):
    import torch
    args = dict(dtype="bf16", batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, l_obs=4, window=8, task=0, top_p=0, max_seqlen=30, budgets=[30] * 2,
                device=torch.device("cpu"))
    args.update(kw)
    return binding.Problem(**args)


def test_keys_and_values_in_another_layout_are_refused():
    """The C side goes by the problem's strides: a tensor that has others would be read, or written, in the wrong places."""
    import torch
    new = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)
    packed = dict(batch=3, budgets=[30] * 3, max_seqlen=12, cu_seqlens=[0, 5, 9, 20])
    q, kv = new(2, 4, 30, 64), new(2, 2, 30, 64)
    good = [(problem(), kv), (problem(), kv.view(-1, 64)), (problem(), new(3, 2, 30, 64)), (problem(), kv.transpose(1, 2)),
            (problem(kv_layout="bnhd"), new(2, 30, 2, 64)), (problem(kv_layout="bnhd"), new(2, 30, 2, 64).transpose(1, 2)),
            (problem(kv_layout="bnhd", batch=1, budgets=[30]), new(1, 31, 2, 64)),
            (problem(n_kv_heads=1), new(2, 1, 30, 64)), (problem(n_kv_heads=1, kv_layout="bnhd"), new(2, 1, 30, 64)),
            (problem(**packed), new(20, 2, 64)), (problem(**packed), new(25, 2, 64)), (problem(**packed), new(20, 2, 64).transpose(0, 1))]
    bad = [(problem(), new(2, 30, 2, 64)), (problem(kv_layout="bnhd"), kv), (problem(), new(1, 2, 30, 64).expand(2, 2, 30, 64)),
           (problem(), new(2, 1, 30, 64).expand(2, 2, 30, 64)), (problem(), new(2, 2, 30, 72)[..., :64]), (problem(), new(2, 2, 31, 64)),
           (problem(), new(2, 2, 31, 64)[:, :, :30]), (problem(), new(2, 2, 29, 64)), (problem(), kv.view(-1, 64)[1:]), (problem(), kv.float()),
           (problem(), new(2, 2, 30, 128)[..., ::2]), (problem(), new(2, 2, 30, 32)),
           (problem(**packed), new(20, 2, 72)[..., :64]), (problem(**packed), new(2, 20, 64)), (problem(**packed), new(19, 2, 64)),
           (problem(**packed), new(1, 2, 64).expand(20, 2, 64)), (problem(**packed), new(20, 1, 64).expand(20, 2, 64))]
    rope = binding.Rope(64, device=torch.device("cpu"))
    for prob, t in good:
        binding.prepare_rotate_prompt(prob, rope, None, t, None, t, stream=0)
    for prob, t in bad:
        ok = next(g for p, g in good if (p.packed, p.shape.stride_h, p.shape.stride_b) == (prob.packed, prob.shape.stride_h, prob.shape.stride_b))
        for k, k_out in ((t, ok), (ok, t)):
            with pytest.raises(ValueError, match="layout expected"):
                binding.prepare_rotate_prompt(prob, rope, None, k, None, k_out, stream=0)
        x = new(20, 4, 64) if prob.packed else q
        for k, v in ((t, ok), (ok, t)):
            with pytest.raises(ValueError, match="layout expected"):
                binding.prepare_attend_prompt(prob, x, k, v, x.clone(), stream=0)


def test_rotated_dimensions_have_a_limit_of_their_own(L):
    """More pairs than a block holds angles for, in heads that have them: a limit, not a wrong shape."""
    c = paged(head_dim=8192, page_stride=2 * 16 * 8192, head_stride=16 * 8192, row_stride=8192)
    st = strides(2 * 3 * 8192, 3 * 8192, 8192)
    s = shape(head_dim=8192, stride_b=2 * 1024 * 8192, stride_h=1024 * 8192, stride_t=8192, q_stride_t=8192)
    for rot, status in ((4098, 9), (8192, 9), (8194, 2), (4097, 2)):
        r = rope(rot_dim=rot)
        assert L.wkv_append_kv_paged(ctypes.byref(c), ctypes.byref(r), P, P, st, None, None, None, P, P, P, 2 * P, None, None, None, None) == status
        assert L.wkv_rotate_prompt(ctypes.byref(s), ctypes.byref(r), None, None, None, P, P, None, None) == status


def test_outputs_whose_rows_share_a_place_are_refused(L):
    """An expanded or overlapping output would be written by several blocks at once."""
    tight = [(3 * 64, 3 * 64, 64), (0, 3 * 64, 64), (4 * 3 * 64, 0, 64), (4 * 3 * 64, 64, 64), (4 * 3 * 64, 3 * 64 - 8, 64), (2 * 3 * 64, 3 * 64, 64)]
    fine = strides(4 * 3 * 64, 3 * 64, 64)
    need = L.wkv_paged_workspace_bytes(ctypes.byref(paged()))
    c, s, r = paged(), shape(max_seqlen=3, l_obs=1, budget=3), rope()
    s2 = shape(max_seqlen=3, l_obs=1, budget=3, batch=2)
    for t in tight:
        assert L.wkv_attend_paged(ctypes.byref(c), P, fine, P, P, P, 2 * P, strides(*t), None, None, None, P, need, None) == 2, t
        assert L.wkv_append_kv_paged(ctypes.byref(c), None, P, P, fine, P, P, strides(*t), None, P, P, 2 * P, None, None, None, None) == 2, t
        assert L.wkv_attend_prompt(ctypes.byref(s2), P, fine, P, P, 2 * P, strides(*t), None, None, None, None) == 2, t
        assert L.wkv_rotate_prompt(ctypes.byref(s2), ctypes.byref(r), P, P, strides(*t), None, None, None, None) == 2, t
    for kw in (dict(stride_b=0), dict(stride_h=0), dict(stride_b=64, stride_h=64), dict(stride_h=64)):
        bad = shape(max_seqlen=3, l_obs=1, budget=3, batch=2, stride_b=2 * 3 * 64, stride_h=3 * 64)
        for name, x in kw.items():
            setattr(bad, name, x)
        assert L.wkv_rotate_prompt(ctypes.byref(bad), ctypes.byref(r), None, None, None, P, P, None, None) == 2, kw
    ptrs = (ctypes.c_void_p * 1)(P)
    for kw in (dict(page_stride=0), dict(head_stride=0), dict(page_stride=16 * 64), dict(head_stride=64), dict(head_stride=2 * 64)):
        bad = paged(**kw)
        assert L.wkv_append_kv_paged(ctypes.byref(bad), None, P, P, fine, None, None, None, None, P, P, 2 * P, None, None, None, None) == 2, kw
        assert L.wkv_evict_kv_paged(ctypes.byref(bad), 1, ptrs, None, 4, None, 0, P, P, P, P, P, P, P, need, None) == 2, kw
    # what lies apart in another order, or has one element, gets as far as the next check
    cu = np.array([0, 1, 3], dtype=np.int32)
    for t in ((64, 3 * 2 * 64, 2 * 64), (3 * 4 * 64, 64, 4 * 64), (4 * 3 * 72, 3 * 72, 72)):
        assert L.wkv_attend_paged(ctypes.byref(c), P, fine, P, P, P, 2 * P, strides(*t), None, None, None, P, need - 1, None) == 5, t
    packed = paged(cu_new_host=cu.ctypes.data, cu_new_dev=P)
    assert L.wkv_attend_paged(ctypes.byref(packed), P, fine, P, P, P, 2 * P, strides(0, 64, 4 * 64), None, None, None, P, 0, None) == 5
    one = paged(batch=1, n_kv_heads=1, n_q_heads=1, max_new=1)
    assert L.wkv_attend_paged(ctypes.byref(one), P, fine, P, P, P, 2 * P, strides(0, 0, 64), None, None, None, P, 0, None) == 5
    # pools that are only read may share rows
    for kw in (dict(page_stride=0), dict(head_stride=0)):
        assert L.wkv_attend_paged(ctypes.byref(paged(**kw)), P, fine, P, P, P, 2 * P, fine, None, None, None, P, 0, None) == 5


def test_tensors_of_another_device_are_refused(monkeypatch):
    """A kernel that is given another device's memory, or the host's, faults: every tensor of a call is looked at."""
    import torch
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    prob, rope = problem(), binding.Rope(64, device=torch.device("cpu"))
    cache = binding.PagedCache(dtype="bf16", batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, num_pages=6,
                               block_table=torch.zeros((2, 3), dtype=i32))
    units, rows = (2, 2), (2, 2, 48)
    zeros = lambda shape, dtype: torch.zeros(shape, dtype=dtype)
    q, kv, pool = (lambda: zeros((2, 4, 30, 64), bf)), (lambda: zeros((2, 2, 30, 64), bf)), (lambda: zeros((6, 2, 16, 64), bf))
    new, newkv, ws = (lambda: zeros((2, 4, 1, 64), bf)), (lambda: zeros((2, 2, 1, 64), bf)), lambda: torch.zeros(cache.workspace_bytes, dtype=torch.uint8)
    calls = [
        (binding.prepare_rotate_prompt, dict(prob=prob, rope=rope), dict(q=q(), k=kv(), q_out=q(), k_out=kv(), positions=zeros((2, 30), i32))),
        (binding.prepare_attend_prompt, dict(prob=prob), dict(q=q(), k=kv(), v=kv(), out=q(), lse=zeros((2, 4, 30), f32), lse_obs=zeros((2, 4, 4), f32),
                                                              status=zeros((1,), i32))),
        (binding.prepare_append_kv_paged, dict(cache=cache, rope=rope),
         dict(k_new=newkv(), v_new=newkv(), lengths=zeros(units, i32), k_pool=pool(), v_pool=pool(), q=new(), q_out=new(), positions=zeros((2, 1), i32),
              lengths_out=zeros(units, i32), row_positions=zeros(rows, i32), row_weights=zeros(rows, f32))),
        (binding.prepare_attend_paged, dict(cache=cache),
         dict(q=new(), k_pool=pool(), v_pool=pool(), lengths=zeros(units, i32), out=new(), workspace=ws(), lse=zeros((2, 4, 1), f32),
              weights_in=zeros(rows, f32), weights_out=zeros(rows, f32))),
        (binding.prepare_evict_kv_paged, dict(cache=cache, budget=3, recent=1),
         dict(k_pools=[pool()], v_pools=[pool()], weights=zeros(rows, f32), positions=zeros(rows, i32), lengths=zeros(units, i32),
              weights_out=zeros(rows, f32), positions_out=zeros(rows, i32), lengths_out=zeros(units, i32), workspace=ws(), budgets=zeros((2,), i32))),
    ]
    away = lambda t: [x.to("meta") for x in t] if isinstance(t, list) else t.to("meta")
    for fn, fixed, tensors in calls:
        fn(**fixed, **tensors, stream=0)
        for name in tensors:
            with pytest.raises(ValueError, match="expected, got one on meta"):
                fn(**fixed, **{**tensors, name: away(tensors[name])}, stream=0)
    with pytest.raises(ValueError, match="on cpu expected, got one on meta"):
        far = binding.Rope(64, device=torch.device("cpu"))
        far.turns = far.turns.to("meta")
        binding.prepare_rotate_prompt(prob, far, q(), None, q(), None, stream=0)
    seed = dict(window_idx=zeros((2, 2, prob.k_max), i32), token_scores=zeros((2, 2, 26), f32), positions=zeros((2, 2, 30), i32), weights=zeros((2, 2, 30), f32))
    for name in seed:
        with pytest.raises(ValueError, match="got one on meta"):
            binding.wkv_seed_rows(prob, **{**seed, name: seed[name].to("meta")}, stream=0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    binding._check_devices(torch.device("cuda", 0), "call", None, 12)
    with pytest.raises(ValueError, match="current device is cuda:0"):
        binding._check_devices(torch.device("cuda", 1), "call")


def test_binding_refuses_status_and_indices_of_other_types():
    import torch
    prob = problem()
    q, kv = torch.zeros((2, 4, 30, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 30, 64), dtype=torch.bfloat16)
    for bad in (torch.zeros(1, dtype=torch.uint8), torch.zeros(1), torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(ValueError, match="status"):
            binding.prepare_attend_prompt(prob, q, kv, kv, q.clone(), status=bad, stream=0)
    binding.prepare_attend_prompt(prob, q, kv, kv, q.clone(), status=torch.zeros(3, dtype=torch.int32)[1:], stream=0)
    with pytest.raises(ValueError, match="None"):
        binding.prepare_attend_prompt(prob, None, kv, kv, q.clone(), stream=0)
    positions = torch.zeros((2, 2, 30), dtype=torch.int32)
    idx = torch.zeros((2, 2, prob.k_max), dtype=torch.int32)
    for bad in (idx.long(), idx[..., :-1].contiguous(), idx.float()):
        with pytest.raises(ValueError, match="window_idx"):
            binding.wkv_seed_rows(prob, bad, None, positions, None, stream=0)
    with pytest.raises(ValueError, match="positions, weights"):
        binding.wkv_seed_rows(prob, idx, None, None, None, stream=0)


def test_binding_takes_a_chunk_of_nothing_without_tensors():
    import torch
    table, n = torch.zeros((2, 4), dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32)
    pool, q = torch.zeros((6, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16)
    args = dict(dtype="bf16", batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, num_pages=6, block_table=table)
    empty, some, dense = (binding.PagedCache(**args, **kw) for kw in (dict(cu_new=[0, 0, 0]), dict(cu_new=[0, 0, 1]), {}))
    ws = empty.alloc_workspace()
    binding.prepare_attend_paged(empty, None, pool, pool, n, None, ws, stream=0)
    binding.prepare_append_kv_paged(empty, None, None, n, pool, pool.clone(), stream=0)
    for cache in (some, dense):
        for q_, out in ((None, q), (q, None)):
            with pytest.raises(ValueError, match="expected, got"):
                binding.prepare_attend_paged(cache, q_, pool, pool, n, out, ws, stream=0)
