"""CPU-only checks of the rows in front of a draft and of a layer against its cache: struct mirrors and refusals before any device work."""
import ctypes
import inspect

import pytest
import torch

from paper_2503_17922_b200 import binding, build
from test_cache8_host import NULL, SHAPE, P, P2, P3, P4, draft, layer, paged, ref


@pytest.fixture(scope="module")
def L():
    build.build_library()
    return binding.lib()


def test_struct_mirror_with_rows_before():
    assert ctypes.sizeof(binding.WkvDraftBefore) == 2 * 4 + 2 * 8
    assert binding.WkvDraftBefore.before.offset == ctypes.sizeof(binding.WkvDraft) == 16


def whole(**kw):
    x = binding.WkvDraftBefore(ctypes.sizeof(binding.WkvDraftBefore), 1, P, P2)
    for k, v in kw.items():
        setattr(x, k, v)
    return x


def test_keep_refuses_lengths_out_in_the_place_of_before(L):
    two = (ctypes.c_void_p * 2)(P3, P4)
    keep = lambda d, out: L.wkv_keep_draft_paged(ref(paged()), ref(d), 2, two, two, P, P, out, None, None, None)
    assert keep(whole(), P2) == SHAPE and keep(whole(), P) == SHAPE
    assert L.wkv_keep_draft_paged8(ref(paged()), ref(whole()), 1, ref(layer()), P, P, P2, None, None, None) == SHAPE
    assert keep(whole(struct_size=20), P2) == SHAPE and keep(whole(struct_size=32), P3) == SHAPE
    assert keep(whole(masks=None), P3) == NULL


def test_a_tensor_given_twice_is_refused(L):
    """Rows are moved inside every tensor, by blocks of its own: the same one twice would be moved by two at once."""
    c, BIG = paged(), 1 << 40
    ptrs = lambda *p: (ctypes.c_void_p * len(p))(*p)
    keep = lambda k, v: L.wkv_keep_draft_paged(ref(c), ref(draft()), len(k), k, v, P, P, P2, None, None, None)
    assert keep(ptrs(P), ptrs(P)) == SHAPE and keep(ptrs(P, P2), ptrs(P3, P)) == SHAPE and keep(ptrs(P, P), None) == SHAPE
    P5, P6 = 0x5000, 0x6000
    other = lambda **kw: layer(**{**dict(k_codes=P5, v_codes=P6, k_scales=P5, v_scales=P6), **kw})
    for second in (layer(), other(k_codes=P), other(v_codes=P), other(k_scales=P4), other(v_scales=P4)):
        two = (binding.WkvCache8 * 2)(layer(), second)
        assert L.wkv_keep_draft_paged8(ref(c), ref(draft()), 2, two, P, P, P2, None, None, None) == SHAPE
        assert L.wkv_evict_kv_paged8(ref(c), 2, two, 5, None, 0, P, P, P, P, P, P, P, BIG, None) == SHAPE
        assert b"are the same" in L.wkv_last_error_detail()


def test_a_layer_is_held_against_the_cache_of_every_call(L):
    """A description with more pages, heads, rows or columns than the layer's pools have, other strides or another type is refused by every call that takes the
    layer (on CPU tensors: a call that was not would go on to the library); one that differs in the new tokens alone is not."""
    def describe(kind="i8", pages=20, hk=2, d=64, page=16, max_new=3, layout="phsd", cls=binding.PagedCache8):
        kw = dict(kind=kind) if cls is binding.PagedCache8 else {}
        return cls(dtype="bf16", batch=2, n_q_heads=4, n_kv_heads=hk, head_dim=d, page_size=page, num_pages=pages, max_new=max_new, layout=layout,
                   block_table=torch.zeros((2, 9), dtype=torch.int32), **kw)
    made = describe()
    codes = [torch.zeros((20, 2, 16, 64), dtype=torch.uint8) for _ in range(2)]
    one = binding.Layer8(made, *codes, made.alloc_scales(), made.alloc_scales())
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    ws = torch.zeros(10, dtype=torch.uint8)

    def calls(c):
        hk, d, m, cap = c.shape.n_kv_heads, c.shape.head_dim, c.shape.max_new, c.capacity
        bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
        k, q, lengths, masks = bf(2, hk, m, d), bf(2, 4, m, d), ints(2, hk), ints(2, m, 1)
        weights = lambda: torch.zeros((2, hk, cap))
        return [lambda: binding.prepare_append_kv_paged8(c, one, k, k, lengths, stream=0), lambda: binding.prepare_attend_paged8(c, one, q, lengths, q.clone(), ws, stream=0),
                lambda: binding.prepare_read_kv_paged8(c, one, lengths, bf(2, hk, 5, d), None, stream=0),
                lambda: binding.wkv_evict_kv_paged8(c, [one, one], weights(), ints(2, hk, cap), lengths, 5, 0, weights(), ints(2, hk, cap), ints(2, hk), ws),
                lambda: binding.wkv_keep_draft_paged8(c, masks, [one], ints(2), lengths, ints(2, hk))]
    others = [describe("e4m3"), describe(pages=21), describe(hk=4), describe(d=128), describe(page=32), describe(layout=(2 * 16 * 64, 16 * 64, 80)),
              describe(layout=(2 * 16 * 64 + 64, 16 * 64, 64)), describe(cls=binding.PagedCache)]
    for i, c in enumerate(others):
        for j, call in enumerate(calls(c)):
            with pytest.raises(ValueError):
                call()
                pytest.fail(f"description {i}, call {j} was not refused")
    for c in (made, describe(max_new=7), describe(layout="pshd")):         # (the last: as many bytes)
        one.check(c)
        for call in calls(c)[:3]:
            assert isinstance(call(), binding.PreparedCall)


def test_the_gather_holds_its_layers_against_the_cache(L):
    table = torch.zeros((1, 9), dtype=torch.int32)
    make = lambda pages: binding.PagedCache8(kind="i8", dtype="bf16", batch=1, n_q_heads=2, n_kv_heads=2, head_dim=64, page_size=16, num_pages=pages, block_table=table)
    cache, larger = make(9), make(10)
    one = binding.Layer8(cache, *(torch.zeros((9, 2, 16, 64), dtype=torch.uint8) for _ in range(2)), cache.alloc_scales(), cache.alloc_scales())
    prob = binding.Problem(dtype="bf16", batch=1, n_q_heads=2, n_kv_heads=2, head_dim=64, l_obs=8, window=8, task=0, top_p=0, max_seqlen=100, budgets=[40], device="cpu")
    k, idx = torch.zeros((1, 2, 100, 64), dtype=torch.bfloat16), torch.zeros((1, 2, prob.k_max), dtype=torch.int32)
    assert isinstance(binding.prepare_gather_kv_paged8(prob, cache, [one], [k], [k], idx, stream=0), binding.PreparedCall)
    with pytest.raises(ValueError):
        binding.prepare_gather_kv_paged8(prob, larger, [one], [k], [k], idx, stream=0)


def test_python_face_refuses_other_rows_before(L):
    table = torch.zeros((2, 9), dtype=torch.int32)
    kw = dict(dtype="bf16", batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, num_pages=20, block_table=table, max_new=3)
    cache, plain = binding.PagedCache8(kind="i8", **kw), binding.PagedCache(**kw)
    codes = [torch.zeros((20, 2, 16, 64), dtype=torch.uint8) for _ in range(2)]
    one = binding.Layer8(cache, *codes, cache.alloc_scales(), cache.alloc_scales())
    pools = [torch.zeros((20, 2, 16, 64), dtype=torch.bfloat16) for _ in range(2)]
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    q, masks, ws, lengths = torch.zeros((2, 4, 3, 64), dtype=torch.bfloat16), ints(2, 3, 1), torch.zeros(10, dtype=torch.uint8), ints(2, 2)
    for before in (ints(2), ints(2, 2).long(), ints(2, 2).to("meta")):
        with pytest.raises(ValueError):
            binding.prepare_attend_draft_paged(plain, masks, q, *pools, lengths, q.clone(), ws, before=before)
        with pytest.raises(ValueError):
            binding.prepare_attend_paged8(cache, one, q, lengths, q.clone(), ws, draft=masks, before=before)
        with pytest.raises(ValueError):
            binding.wkv_keep_draft_paged(plain, masks, pools[:1], pools[1:], ints(2), lengths, ints(2, 2), before=before)
        with pytest.raises(ValueError):
            binding.wkv_keep_draft_paged8(cache, masks, [one], ints(2), lengths, ints(2, 2), before=before)
    with pytest.raises(ValueError):
        binding.prepare_attend_paged8(cache, one, q, lengths, q.clone(), ws, before=lengths)


@pytest.mark.parametrize("call", [binding.prepare_attend_draft_paged, binding.prepare_attend_paged8, binding.wkv_keep_draft_paged, binding.wkv_keep_draft_paged8])
def test_rows_before_come_behind_every_argument_that_was_there(call):
    """A stream that is given by its place stays the stream."""
    assert list(inspect.signature(call).parameters)[-2:] == ["stream", "before"]
