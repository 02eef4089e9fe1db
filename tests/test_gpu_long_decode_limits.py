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
