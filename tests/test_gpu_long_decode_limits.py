"""Limits of the calls of a long decode: memory that they share with one another, numbers at the ends of the 4-bit format,
layouts that are the same memory."""
import math

import pytest
import torch

import paper_2608_13226_gb300 as cp
from test_gpu_long_decode import Cache, I4, _lib, bits, ints  # noqa: F401
from test_gpu_serve import BF16, F32, gen, randn

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ memory of two tensors
def test_weights_beside_and_in_place_of_others():
    """Rows of weights between rows of queries and outputs are taken; in their place, the workspace's or the lengths' they are refused."""
    B, Hq, H, D = 3, 4, 2, 64
    c = Cache(gen(0), B, 64, 16, H, D, F32)
    keys, lens = c.W * 16, ints([64, 30, 1])
    x = randn(gen(1), B, 2 * Hq * D + keys, dtype=F32)
    q, out, w = x[:, :Hq * D].view(B, Hq, D), x[:, Hq * D:2 * Hq * D].view(B, Hq, D), x[:, 2 * Hq * D:]
    w.zero_()
    alone = torch.zeros(B, keys, device="cuda")
    want = cp.coverprune_decode_attention(q.clone(), c.k, c.v, c.table, lens, weight=alone)
    cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, weight=w, out=out)
    assert torch.equal(out, want["out"]) and torch.equal(w, alone)
    ws = want["ws"]
    words = ws[:ws.numel() // 4 * 4].view(F32)
    for kw in (dict(weight=out[:, 0], out=out), dict(weight=x[:, 2 * Hq * D - 4:-4], out=out), dict(weight=q[:, 0]), dict(weight=words[:B * keys].view(B, keys), ws=ws),
               dict(weight=words[-B * keys:].view(B, keys), ws=ws)):
        before = kw["weight"].clone()
        with pytest.raises(cp.CoverPruneError) as e:
            cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, **kw)
        assert e.value.status == cp.CP_EINVAL and torch.equal(bits(kw["weight"]), bits(before))
    both = torch.zeros(B * keys, device="cuda")
    with pytest.raises(cp.CoverPruneError):
        cp.coverprune_decode_attention(q, c.k, c.v, c.table, both.view(torch.int32)[5:5 + B], weight=both.view(B, keys))


def test_evict_weights_between_one_anothers_rows():
    """Old and new weights of a sequence side by side in one tensor share nothing."""
    c, lens = Cache(gen(0), 3, 64, 16, 1, 64, BF16), ints([64, 40, 7])
    other = Cache(gen(0), 3, 64, 16, 1, 64, BF16)
    x = torch.rand(3, 2, c.W * 16, generator=gen(1), device="cuda")
    w = x[:, 0].clone()
    want = cp.coverprune_cache_evict(other.k, other.v, other.table, lens, w, 20, first=2, recent=3)
    r = cp.coverprune_cache_evict(c.k, c.v, c.table, lens, x[:, 0], 20, first=2, recent=3, new_weight=x[:, 1])
    assert torch.equal(x[:, 0], w) and torch.equal(x[:, 1], want["weight"]) and torch.equal(r["kept"], want["kept"])
    assert torch.equal(c.k, other.k) and torch.equal(c.v, other.v)
    turns = torch.rand(3, 2 * c.W * 16, device="cuda")  # rows that take turns, but a word too near
    with pytest.raises(cp.CoverPruneError) as e:
        cp.coverprune_cache_evict(c.k, c.v, c.table, lens, turns[:, :c.W * 16], 20, new_weight=turns[:, c.W * 16 - 1:-1])
    assert e.value.status == cp.CP_EINVAL


# ------------------------------------------------------------------ one memory, two descriptions
@pytest.mark.parametrize("Hq,H,D", [(28, 4, 128), (20, 20, 64), (64, 4, 128)])
def test_pages_of_one_row(Hq, H, D):
    """The rows of pages of 16 are pages of one as well: the same memory in the same order, dealt out alike, and so the same bits."""
    B, keys = 9, 4096
    c = Cache(gen(D), B, keys, 16, H, D, I4)
    lens, q = ints([keys - 100 * b for b in range(B)]), randn(gen(1), B, Hq, D, dtype=BF16)
    single = (c.table[:, :, None] * 16 + torch.arange(16, device="cuda", dtype=torch.int32)).reshape(B, -1)
    # the dimension of one has no stride that counts, whatever the tensor's says
    k, v, kb, vb = (t.reshape(-1, 1, *t.shape[2:]) for t in (c.k, c.v, c.kb, c.vb))
    w, w1 = torch.zeros(2, B, keys, device="cuda")
    for weight in (False, True):
        want = cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, lse=True, weight=w if weight else None, **c.kw)
        got = cp.coverprune_decode_attention(q, k, v, single, lens, lse=True, weight=w1 if weight else None, k_block=kb, v_block=vb)
        assert torch.equal(bits(got["out"]), bits(want["out"])) and torch.equal(got["lse"], want["lse"])
    assert torch.equal(w, w1)
