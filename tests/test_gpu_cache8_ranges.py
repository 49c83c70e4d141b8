"""GPU tests of attention over the 8-bit cache and of drafts where values differ by far in size, each against a reference in 64 bits."""
import pytest
import torch

import cache8_util as cu
import operators_util as ou
from paper_2503_17922_b200 import binding as wkv
from test_gpu_cache8 import Attend, gen, random_tree

pytestmark = pytest.mark.gpu


# ---- values of very different sizes --------------------------------------------------------------
class Far(Attend):
    """A bf16 query's weights p_j 2^e_j are f16 numbers on the warp-level kernel, times 2^14 / V with a power of two V <= max_j p_j 2^e_j over the keys that
    the row sees.  f16 has steps of 2^-24 at least, so a weight is off by 2^-25 V / 2^14 = 2^-39 V at most where it is below f16's normal numbers (above them
    it is half_step(f16) of itself, less than the half_step(bf16) of the common bound).  An element that the large value's code leaves at 0, or nearly, is off by
    that much of the others' codes: 2^-39 max_j(p_j 2^e_j) sum_j |code_jc|, with the last rounding's 1 + r."""

    def check(self):
        torch.cuda.synchronize()
        r = ou.half_step(self.dtype)
        n, m, G = int(self.lengths[0, 0]), self.news[0], self.hq
        (k, _), (v, _) = self.rows(0, 0, 0, n), self.rows(1, 0, 0, n)
        scales = cu.powers(self.c.raw(0, 1, 0, 0, n)[1].int() - 127)
        for head in range(G):
            ref, lse, p, bd = cu.attention_seen(self.part(self.q, 0, head), k, v, self.seen(0, 0))
            least = 2.0 ** -39 * (p * scales).amax(1, keepdim=True) * (v / scales[:, None]).abs().sum(0) if self.dtype == torch.bfloat16 else 0.0
            ou.assert_close(self.part(self.out, 0, head), ref, ou.output_bound(ref, bd, self.dtype) + least * (1 + r), f"out {head}")
            ou.assert_close(self.lse[0, head, :m], lse, ou.lse_bound(lse, bd), f"lse {head}")
        assert wkv.device_status(self.ws) == 0


def rescale(a, kv, row, byte):
    """The scale byte of a row of a's only unit."""
    n = int(a.lengths[0, 0])
    codes, scales, _ = a.c.raw(0, kv, 0, 0, n)
    scales[row] = byte
    a.c.put(0, kv, 0, 0, torch.arange(n), codes, scales)


# rows of up to 64, and what is left to the same kernel beyond: d above 128, pages that eight does not divide; the others, which are to agree
HIDDEN = [("bf16", 64, 1, 2, 16), ("bf16", 128, 4, 2, 16), ("bf16", 128, 4, 4, 16), ("bf16", 128, 4, 16, 16), ("bf16", 256, 4, 10, 16), ("bf16", 256, 4, 40, 16),
          ("bf16", 128, 4, 40, 6), ("bf16", 128, 4, 40, 16), ("f32", 128, 4, 6, 16)]


@pytest.mark.parametrize("dtype,d,G,new,page", HIDDEN)
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("e", [45, 60, 100])
def test_a_large_value_of_a_later_token(dtype, d, G, new, page, kind, e):
    """A finite value 2^e times the others' size: the queries in front of it give the same bits as without it, those behind it what it weighs."""
    a = Far(dtype, kind, G, 1, d, page, "phsd", [[300]], [new], False)
    a.run()
    a.check()
    clean, clean_lse = a.out.clone(), a.lse.clone()
    rescale(a, 1, 300 - new + new // 2, min(120 + e, 227))
    a.run()
    a.check()
    i = new // 2
    assert torch.equal(a.out[0, :, :i], clean[0, :, :i]) and torch.equal(a.lse, clean_lse)
    assert not torch.equal(a.out[0, :, i:], clean[0, :, i:])


@pytest.mark.parametrize("dtype,d,new", [("bf16", 128, 2), ("bf16", 64, 4), ("bf16", 128, 15), ("bf16", 256, 9), ("bf16", 128, 40), ("f32", 64, 7)])
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_a_large_value_of_another_branch(dtype, d, new, kind):
    sees = cu.tree_of(random_tree(gen(5), new, 0.3))
    token = next(t for t in range(new - 1, -1, -1) if not sees[:, t].all())
    a = Far(dtype, kind, 4, 1, d, 16, "phsd", [[200]], [new], False, sees=[sees])
    a.run()
    a.check()
    clean = a.out.clone()
    rescale(a, 1, 200 - new + token, 187)
    a.run()
    a.check()
    on = sees[:, token].cuda()
    assert torch.equal(a.out[0][:, ~on], clean[0][:, ~on]) and not torch.equal(a.out[0][:, on], clean[0][:, on])


@pytest.mark.parametrize("dtype,d,new", [("bf16", 128, 1), ("bf16", 64, 1), ("bf16", 128, 4), ("bf16", 256, 1), ("bf16", 256, 20), ("bf16", 128, 40), ("f32", 128, 2)])
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("at", [3, 150, 250])
def test_a_large_value_of_next_to_no_weight(dtype, d, new, kind, at):
    """A key that all see, with a value of 2^60 and a weight of 2^-88 at most (logits of q sqrt(d) elsewhere and of -8 q sqrt(d) at the key, 9 q sqrt(d) / ln 2
    bits apart: 104, 88 and 125): what it adds is far below the others' rounding, and they keep their bits."""
    a = Far(dtype, kind, 4, 1, d, 16, "phsd", [[300]], [new], False)
    codes, scales, _ = a.c.raw(0, 0, 0, 0, 300)
    codes.fill_(0x68 if kind == "e4m3" else 64)                           # 64
    codes[at] = 0xe8 if kind == "e4m3" else 256 - 64
    scales.fill_(121)                                                     # times 2^-6
    scales[at] = 124                                                     # minus 8
    a.c.put(0, 0, 0, 0, torch.arange(300), codes, scales)
    a.q.fill_(0.6 if d >= 128 else 1.0)
    rescale(a, 1, at, 187)
    a.run()
    a.check()
