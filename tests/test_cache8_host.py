"""CPU-only checks of the norms with rotary positions, the 8-bit cache and the drafts: struct mirrors and refusals before any device work."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2503_17922_b200 import binding, build

NULL, SHAPE, DTYPE, BUDGET, WORKSPACE, ALIGN, UNSUPPORTED, LIMIT = 1, 2, 3, 4, 5, 6, 7, 9
P, P2, P3, P4 = 0x1000, 0x2000, 0x3000, 0x4000      # aligned addresses that nothing follows: every call here is refused on the host
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    build.build_library()
    lib = binding.lib()
    lib.launched_before = lib.wkv_launch_count()
    return lib


def of(cls, base, kw):
    x = cls()
    x.struct_size = ctypes.sizeof(cls)
    for k, v in {**base, **kw}.items():
        setattr(x, k, v)
    return x


def shape(**kw):
    return of(binding.WkvShape, dict(dtype=binding.WKV_BF16, batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, l_obs=8, window=8, max_seqlen=1024, budget=128,
                                     stride_b=2 * 1024 * 64, stride_h=1024 * 64, stride_t=64, q_stride_b=4 * 8 * 64, q_stride_h=8 * 64, q_stride_t=64), kw)


def paged(**kw):
    return of(binding.WkvPaged, dict(dtype=binding.WKV_BF16, batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, max_new=3, page_size=16, num_pages=20,
                                     max_pages=9, block_table=P, page_stride=2 * 16 * 64, head_stride=16 * 64, row_stride=64), kw)


def rope(**kw):
    return of(binding.WkvRope, dict(rot_dim=64, scale=1.0, turns=P), kw)


def norm(**kw):
    return of(binding.WkvHeadNorm, dict(eps=1e-6, q_weight=P, k_weight=P), kw)


def axes(**kw):
    return of(binding.WkvRopeAxes, dict(n_axes=3, axis=P, position_stride=4096), kw)


def layer(**kw):
    return of(binding.WkvCache8, dict(type=0, k_codes=P, v_codes=P2, k_scales=P3, v_scales=P4), kw)


def draft(**kw):
    return of(binding.WkvDraft, dict(words=1, masks=P), kw)


def strides(*st):
    return (ctypes.c_int64 * 3)(*st)


QS, KS, NS = strides(4 * 1024 * 64, 1024 * 64, 64), strides(2 * 3 * 64, 3 * 64, 64), strides(4 * 3 * 64, 3 * 64, 64)
ref = ctypes.byref


def test_struct_mirrors():
    assert ctypes.sizeof(binding.WkvHeadNorm) == 4 * 4 + 2 * 8
    assert ctypes.sizeof(binding.WkvRopeAxes) == 2 * 4 + 2 * 8
    assert ctypes.sizeof(binding.WkvCache8) == 2 * 4 + 4 * 8
    assert ctypes.sizeof(binding.WkvDraft) == 2 * 4 + 8


def rotate(L, s=None, n=None, r=None, x=None, q=P, q_out=P2, qs=QS, k=P3, k_out=P4, positions=P):
    return L.wkv_norm_rotate_prompt(ref(s or shape()), n and ref(n), r and ref(r), x and ref(x), q, q_out, qs, k, k_out, positions, None)


@pytest.mark.parametrize("kw,want", [
    (dict(), NULL), (dict(n=norm(struct_size=4)), SHAPE), (dict(n=norm(eps=-1.0)), SHAPE), (dict(n=norm(eps=float("nan"))), SHAPE),
    (dict(n=norm(eps=float("inf"))), SHAPE), (dict(n=norm(offset=float("nan"))), SHAPE), (dict(n=norm(reserved=1)), SHAPE), (dict(r=rope(rot_dim=3)), SHAPE),
    (dict(r=rope(rot_dim=66)), SHAPE), (dict(r=rope(turns=None)), NULL), (dict(r=rope(), x=axes(struct_size=8)), SHAPE), (dict(r=rope(), x=axes(n_axes=0)), SHAPE),
    (dict(r=rope(), x=axes(position_stride=2047)), SHAPE), (dict(r=rope(), x=axes(axis=None)), NULL), (dict(r=rope(), x=axes(), positions=None), NULL),
    (dict(n=norm(), x=axes()), SHAPE), (dict(n=norm(), q=None), NULL), (dict(n=norm(), q=None, q_out=None, k=None, k_out=None), NULL),
    (dict(n=norm(), q=P + 2), ALIGN), (dict(n=norm(), qs=strides(64, 64, 32)), SHAPE), (dict(n=norm(), qs=strides(0, 1024 * 64, 64)), SHAPE),
    (dict(n=norm(), s=shape(head_dim=264, stride_t=264, stride_h=1024 * 264, stride_b=2 * 1024 * 264, q_stride_t=264, q_stride_h=8 * 264, q_stride_b=32 * 264)), UNSUPPORTED), (dict(n=norm(), s=shape(struct_size=3)), SHAPE),
])
def test_rotate_refusals(L, kw, want):
    assert rotate(L, **kw) == want


def append(L, c=None, lay=None, n=None, r=None, x=None, k=P, v=P2, ks=KS, q=None, q_out=None, qs=NS, positions=P, lengths=P, k_pool=P3, v_pool=P4, out=P2,
           rp=None, rw=None, eight=True):
    turn = (n and ref(n), r and ref(r), x and ref(x))
    if eight:
        return L.wkv_append_kv_paged8(ref(c or paged()), ref(lay or layer()), *turn, k, v, ks, q, q_out, qs, positions, lengths, out, rp, rw, None)
    return L.wkv_norm_append_kv_paged(ref(c or paged()), *turn, k, v, ks, q, q_out, qs, positions, lengths, k_pool, v_pool, out, rp, rw, None)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("kw,want", [
    (dict(n=norm(eps=-1.0)), SHAPE), (dict(r=rope(order=2)), SHAPE), (dict(r=rope(), x=axes(position_stride=5)), SHAPE), (dict(r=rope(), positions=None), NULL),
    (dict(n=norm(), k=None), NULL), (dict(n=norm(), v=P + 8), ALIGN), (dict(n=norm(), ks=strides(0, 1, 64)), ALIGN), (dict(n=norm(), q=P), NULL),
    (dict(n=norm(), q=P, q_out=P, qs=strides(0, 3 * 64, 64)), SHAPE), (dict(n=norm(), lengths=None), NULL), (dict(n=norm(), out=P), SHAPE),
    (dict(n=norm(), positions=None, rp=P), NULL), (dict(n=norm(), c=paged(head_dim=272, row_stride=272, head_stride=16 * 272, page_stride=32 * 272)), UNSUPPORTED),
    (dict(n=norm(), c=paged(row_stride=32)), SHAPE), (dict(n=norm(), c=paged(head_stride=64)), SHAPE), (dict(n=norm(), c=paged(block_table=None)), NULL),
])
def test_append_refusals(L, eight, kw, want):
    assert append(L, eight=eight, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(struct_size=8), SHAPE), (dict(type=2), DTYPE), (dict(k_codes=None), NULL), (dict(v_codes=P2 + 8), ALIGN), (dict(k_scales=None), NULL), (dict(v_scales=None), NULL),
    (dict(v_codes=P), SHAPE), (dict(v_scales=P3), SHAPE)])
def test_layer_refusals(L, kw, want):
    bad, c, n = layer(**kw), paged(), 9 * 16
    assert append(L, lay=bad) == want
    assert L.wkv_attend_paged8(ref(c), ref(bad), None, P, NS, P, P2, NS, None, None, None, P, BIG, None) == want
    assert L.wkv_read_kv_paged8(ref(c), ref(bad), None, P, 1, n, P, P2, None) == want
    two = (binding.WkvCache8 * 2)(layer(), bad)
    assert L.wkv_evict_kv_paged8(ref(c), 2, two, 5, None, 0, P, P, P, P, P, P, P, BIG, None) == want
    assert L.wkv_keep_draft_paged8(ref(c), ref(draft()), 2, two, P, P, P2, None, None, None) == want
    ptrs = (ctypes.c_void_p * 2)(P, P2)
    assert L.wkv_gather_kv_paged8(ref(shape()), ref(c), 2, ptrs, ptrs, P, two, None) == want


def test_layers_of_two_types_and_missing_ones(L):
    two = (binding.WkvCache8 * 2)(layer(), layer(type=1))
    c = paged()
    assert L.wkv_evict_kv_paged8(ref(c), 2, two, 5, None, 0, P, P, P, P, P, P, P, BIG, None) == DTYPE
    assert L.wkv_evict_kv_paged8(ref(c), 0, two, 5, None, 0, P, P, P, P, P, P, P, BIG, None) == LIMIT
    assert L.wkv_evict_kv_paged8(ref(c), 33, two, 5, None, 0, P, P, P, P, P, P, P, BIG, None) == LIMIT
    assert L.wkv_evict_kv_paged8(ref(c), 1, None, 5, None, 0, P, P, P, P, P, P, P, BIG, None) == NULL
    assert L.wkv_evict_kv_paged8(ref(c), 1, two, -1, None, 0, P, P, P, P, P, P, P, BIG, None) == BUDGET
    assert L.wkv_evict_kv_paged8(ref(c), 1, two, 5, None, -1, P, P, P, P, P, P, P, BIG, None) == SHAPE
    assert L.wkv_evict_kv_paged8(ref(c), 1, two, 5, None, 0, P, P, P, None, P, P, P, BIG, None) == NULL
    assert L.wkv_evict_kv_paged8(ref(c), 1, two, 5, None, 0, P, P, P, P, P, P, P, 16, None) == WORKSPACE
    assert L.wkv_append_kv_paged8(ref(c), None, None, None, None, P, P2, KS, None, None, None, P, P, None, None, None, None) == NULL


def test_workspace(L):
    c = paged()
    assert L.wkv_paged8_workspace_bytes(ref(c)) > 0
    # rows of codes are multiples of 16 bytes, and at most 256
    assert L.wkv_paged8_workspace_bytes(ref(paged(head_dim=72, row_stride=72, head_stride=16 * 72, page_stride=32 * 72))) == 0
    assert L.wkv_paged_workspace_bytes(ref(paged(head_dim=72, row_stride=72, head_stride=16 * 72, page_stride=32 * 72))) > 0
    assert L.wkv_paged8_workspace_bytes(ref(paged(head_dim=272, row_stride=272, head_stride=16 * 272, page_stride=32 * 272))) == 0
    assert L.wkv_paged8_workspace_bytes(ref(paged(head_stride=16 * 64 + 8))) == 0
    assert L.wkv_paged8_workspace_bytes(ref(paged(dtype=2))) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(s=shape(batch=3)), SHAPE), (dict(s=shape(dtype=0)), SHAPE), (dict(c=paged(n_kv_heads=4)), SHAPE), (dict(idx=None), NULL), (dict(k=None), NULL),
    (dict(c=paged(max_pages=7)), SHAPE), (dict(c=paged(head_stride=64)), SHAPE), (dict(ptrs=(P, P + 4)), ALIGN), (dict(n=0), LIMIT)])
def test_gather_refusals(L, kw, want):
    ptrs = (ctypes.c_void_p * 2)(*kw.get("ptrs", (P, P2)))
    two = (binding.WkvCache8 * 2)(layer(), layer())
    assert L.wkv_gather_kv_paged8(ref(kw.get("s") or shape()), ref(kw.get("c") or paged()), kw.get("n", 2), kw.get("k", ptrs), ptrs, kw.get("idx", P), two, None) == want


@pytest.mark.parametrize("kw,want", [(dict(lengths=None), NULL), (dict(k=None, v=None), NULL), (dict(k=P2), SHAPE), (dict(rows=0), SHAPE), (dict(dtype=2), DTYPE), (dict(k=P + 4), ALIGN)])
def test_read_refusals(L, kw, want):
    assert L.wkv_read_kv_paged8(ref(paged()), ref(layer()), None, kw.get("lengths", P), kw.get("dtype", 1), kw.get("rows", 10), kw.get("k", P), kw.get("v", P2), None) == want


def attend(L, c=None, d=None, q=P, qs=NS, lengths=P, out=P2, os_=NS, wi=None, wo=None, ws=P, n=BIG, eight=True):
    c = c or paged()
    if eight:
        return L.wkv_attend_paged8(ref(c), ref(layer(k_codes=P3, v_codes=P4)), d and ref(d), q, qs, lengths, out, os_, None, wi, wo, ws, n, None)
    return L.wkv_attend_draft_paged(ref(c), d and ref(d), q, qs, P3, P4, lengths, out, os_, None, ws, n, None)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("kw,want", [
    (dict(d=draft(struct_size=8)), SHAPE), (dict(d=draft(words=0)), SHAPE), (dict(d=draft(masks=None)), NULL),
    (dict(d=draft(words=33), c=paged(max_new=1025)), LIMIT), (dict(d=draft(words=1), c=paged(max_new=33)), SHAPE), (dict(d=draft(), q=None), NULL),
    (dict(d=draft(), out=P), SHAPE), (dict(d=draft(), out=P3), SHAPE), (dict(d=draft(), lengths=None), NULL), (dict(d=draft(), n=16), WORKSPACE),
    (dict(d=draft(), ws=P + 16), WORKSPACE), (dict(d=draft(), os_=strides(0, 3 * 64, 64)), SHAPE), (dict(d=draft(), qs=strides(1, 1, 1)), ALIGN),
    (dict(d=draft(), c=paged(head_dim=320, row_stride=320, head_stride=16 * 320, page_stride=32 * 320)), UNSUPPORTED)])
def test_attend_refusals(L, eight, kw, want):
    assert attend(L, eight=eight, **kw) == want


def test_attend_other_refusals(L):
    assert attend(L, eight=False) == NULL                                 # without a draft
    assert attend(L, d=draft(), wi=P, wo=P) == UNSUPPORTED
    assert attend(L, d=draft(), wo=P) == UNSUPPORTED
    assert attend(L, wi=P) == NULL


def test_draft_refusals(L):
    two = (ctypes.c_void_p * 2)(P, P2)
    masks = lambda c=None, parents=P, words=1, m=P2, pos=None: L.wkv_draft_masks(ref(c or paged()), parents, words, m, None, pos, None)
    assert masks(parents=None) == NULL and masks(m=None) == NULL and masks(words=0) == SHAPE and masks(c=paged(max_new=33)) == SHAPE
    assert masks(c=paged(max_new=2000), words=64) == LIMIT and masks(pos=P) == SHAPE
    keep = lambda c=None, d=None, n=2, k=two, v=two, last=P, lengths=P, out=P2: L.wkv_keep_draft_paged(
        ref(c or paged()), d and ref(d), n, k, v, last, lengths, out, None, None, None)
    assert keep() == NULL and keep(d=draft(), n=0) == LIMIT and keep(d=draft(), n=33) == LIMIT and keep(d=draft(), k=None) == NULL
    assert keep(d=draft(), last=None) == NULL and keep(d=draft(), out=P) == SHAPE and keep(d=draft(words=0)) == SHAPE
    assert keep(d=draft(), c=paged(head_stride=64)) == SHAPE and keep(d=draft(), c=paged(max_new=1025, max_pages=70)) == LIMIT
    wide = paged(head_dim=1024, row_stride=1024, head_stride=16 * 1024, page_stride=32 * 1024)
    assert keep(d=draft(), c=wide) == LIMIT


def test_nothing_was_launched(L):
    assert L.wkv_launch_count() == L.launched_before


def test_python_face_refuses(L):
    """Shapes, types and devices, which the C side cannot see (on CPU tensors: every call is refused, or would be, before the library is reached)."""
    table = torch.zeros((2, 9), dtype=torch.int32)
    kw = dict(dtype="bf16", batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, num_pages=20, block_table=table, max_new=3)
    cache = binding.PagedCache8(kind="i8", **kw)
    with pytest.raises(KeyError):
        binding.PagedCache8(kind="e5m2", **kw)
    codes, scales = torch.zeros((20, 2, 16, 64), dtype=torch.uint8), torch.zeros((20, 2, 16), dtype=torch.uint8)
    one = binding.Layer8(cache, codes, codes.clone(), scales, scales.clone())
    for args in ((codes[:19].clone(), codes, scales, scales), (codes.short(), codes, scales, scales), (codes, codes, scales[:, :, :8], scales), (codes, codes, scales.int(), scales)):
        with pytest.raises(ValueError):
            binding.Layer8(cache, *args)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    q, k, lengths, ws = bf(2, 4, 3, 64), bf(2, 2, 3, 64), ints(2, 2), torch.zeros(10, dtype=torch.uint8)
    bad = [lambda: binding.prepare_append_kv_paged8(cache, one, k[:, :1], k, lengths), lambda: binding.prepare_append_kv_paged8(cache, one, k.float(), k, lengths),
           lambda: binding.prepare_append_kv_paged8(cache, one, k, k, ints(2, 3)), lambda: binding.prepare_append_kv_paged8(cache, one, k, k, lengths, positions=ints(7)),
           lambda: binding.prepare_append_kv_paged8(cache, one, k, k, lengths, norm=binding.HeadNorm(torch.ones(64))),
           lambda: binding.prepare_append_kv_paged8(cache, one, k, k, lengths, norm=binding.HeadNorm(bf(32))),
           lambda: binding.prepare_append_kv_paged8(cache, one, k, k, lengths, axes=binding.RopeAxes([0], 2, device="cpu"), positions=ints(2, 2, 3)),
           lambda: binding.RopeAxes([0, 2], 2, device="cpu"), lambda: binding.HeadNorm(bf(2, 64)),
           lambda: binding.prepare_read_kv_paged8(cache, one, lengths, None, None), lambda: binding.prepare_read_kv_paged8(cache, one, lengths, bf(2, 2, 5, 32), None),
           lambda: binding.prepare_read_kv_paged8(cache, one, lengths, bf(2, 2, 5, 64), bf(2, 2, 6, 64)), lambda: binding.prepare_read_kv_paged8(cache, one, lengths, q.half(), None),
           lambda: binding.prepare_attend_paged8(cache, one, q[:, :2], lengths, q, ws), lambda: binding.prepare_attend_paged8(cache, one, q, lengths, q.clone(), ws, draft=ints(2, 3)),
           lambda: binding.prepare_attend_paged8(cache, one, q, lengths, q.clone(), ws, draft=ints(2, 4, 1)), lambda: binding.prepare_attend_paged8(cache, one, q, lengths, q.clone(), ws, lse=torch.zeros(2, 4, 2)),
           lambda: binding.wkv_draft_masks(cache, ints(2, 4), ints(2, 3, 1)), lambda: binding.wkv_draft_masks(cache, ints(2, 3).long(), ints(2, 3, 1)),
           lambda: binding.wkv_keep_draft_paged8(cache, ints(2, 3, 1), [one], ints(3), lengths, lengths.clone()),
           lambda: binding.wkv_evict_kv_paged8(cache, [one], torch.zeros(2, 2, 144), ints(2, 2, 143), lengths, 5, 0, torch.zeros(2, 2, 144), ints(2, 2, 144), ints(2, 2), ws),
           lambda: binding.prepare_append_kv_paged8(cache, one, k, k, lengths.to("meta"))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    # the device's own refusal reaches Python with its reason: rows that lie in one place
    with pytest.raises(binding.WkvError) as e:
        binding.prepare_attend_paged8(cache, one, q, lengths, q, ws, stream=0).run()
    assert e.value.status == SHAPE and "out" in str(e.value)
    assert np.prod(one.tensors[0].shape) == 20 * 2 * 16 * 64
