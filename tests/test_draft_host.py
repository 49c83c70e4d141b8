"""CPU-only checks of the rows in front of a draft and of a layer against its cache: struct mirrors and refusals before any device work."""
import ctypes

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
