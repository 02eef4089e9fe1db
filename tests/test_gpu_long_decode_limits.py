"""Limits of the calls of a long decode: memory that they share with one another, numbers at the ends of the 4-bit format,
layouts that are the same memory."""
import pytest
import torch

import paper_2608_13226_gb300 as cp
from test_gpu_long_decode import I4, Cache, _lib, as_fours, attention, bits, ints  # noqa: F401
from test_gpu_serve import BF16, F32, assert_stored, gen, randn, wide

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


# ------------------------------------------------------------------ 4 bits at the ends of their scales
def check_codes(x, head, dtype):
    """Codes and scales of rows x [T, H, D] are those of the definition, an operation of float32 at a time: bit for bit."""
    x = x.to(dtype)
    T, H, D = x.shape
    c = Cache(gen(0), 1, T, 16, H, D, I4)
    st, head = ints([0, T]), None if head is None else torch.tensor(head, device="cuda")
    cp.coverprune_cache_append(x, x.flip(0), c.k, c.v, c.table, ints([0]), starts=st, k_scale=head, v_scale=head, **c.kw)
    j = torch.arange(T, device="cuda")
    at = (c.table[0].long()[j // 16], j % 16)
    for cache, blocks, rows in ((c.k, c.kb, x), (c.v, c.vb, x.flip(0))):
        codes, scale = as_fours(rows.float(), head)
        held = bits(cache)[at]
        assert torch.equal(bits(blocks)[at][..., :D // 16], bits(scale))
        assert torch.equal(torch.stack([held & 15, held >> 4], -1).flatten(-2).float() - 8, codes)
        assert bool((bits(blocks)[at][..., D // 16:] == 0).all())
    return scale.float(), codes


def blocks_up_to(g, T, H, D, lo, hi, head):
    """Rows whose blocks' largest component is 7 h 2^e with e spread over lo to hi: mixed components, some zero, the largest anywhere."""
    x = 2 * torch.rand(T, H, D // 16, 16, generator=g, device="cuda", dtype=torch.float64) - 1
    x[torch.rand(x.shape, generator=g, device="cuda") < 0.1] = 0
    x /= x.abs().amax(-1, keepdim=True)
    top = 2.0 ** (lo + (hi - lo) * torch.rand(T, H, D // 16, 1, generator=g, device="cuda", dtype=torch.float64))
    h = torch.ones(H, dtype=torch.float64) if head is None else torch.tensor(head, dtype=torch.float64)
    return (x * top * 7 * h.cuda()[:, None, None]).flatten(-2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,head", [(64, None), (96, [0.3, 1.7]), (32, [-0.7, 2.0 ** -9])])
def test_codes_of_small_and_large_scales(dtype, D, head):
    g = gen(D)
    s, n = check_codes(blocks_up_to(g, 700, 2, D, -11.0, -5.9, head), head, dtype)  # subnormal scales: 0 to 8 steps of 2^-9
    small = (s.abs() > 0) & (s.abs() < 2.0 ** -6)
    assert bool((s == 0).any()) and bool(small.any()) and (n.abs().unflatten(-1, (-1, 16)) == 7).sum(-1)[small].max() > 2  # clipped ones
    if head is None or min(head) > 0:  # a negative factor makes scales negative, which the definition does not bound
        s, n = check_codes(blocks_up_to(g, 700, 2, D, 8.5, 14.0, head), head, dtype)  # 448 at most: what is beyond 7 of it is 7
        full = n.unflatten(-1, (-1, 16))[s == 448.0]
        assert len(full) > 100 and len(full.unique()) == 15
    check_codes(blocks_up_to(g, 700, 2, D, -6.01, -5.99, head), head, dtype)
    check_codes(blocks_up_to(g, 700, 2, D, 8.8, 8.81, [abs(h) for h in head] if head else None), [abs(h) for h in head] if head else None, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("head", [[1e-17, 1e-30], [2e-38, 1e-35], [1e16, 3e30], [3e-16, 5e13], [1e38, 1e-37]])
def test_codes_of_far_steps(dtype, head):
    """Steps below 1e-15 and above 1e15 (and scales whose sevenfold is no float32: all is 0), whole ranges of scales."""
    T = 500
    x = blocks_up_to(gen(1), T, 2, 64, -7.0, 5.0, head)
    x[:, head.index(max(head))].clamp_(-3e38, 3e38)
    s, n = check_codes(x, head, dtype)
    assert len(n[:, 0].unique()) == 15 or head[0] == 1e38


def test_codes_on_borders():
    """Quotients that are halves exactly go to the even one, in the products' way and in the divisions'."""
    half = torch.arange(-15, 16, 2, device="cuda") / 2  # -7.5 .. 7.5
    for s in (2.0 ** -9, 2.0 ** -8, 3 * 2.0 ** -9, 2.0 ** -6, 0.375, 1.0, 208.0, 448.0):
        x = half.clamp(-7, 7).repeat(1, 1, 2)[..., :32] * s
        scale, codes = check_codes(x, None, F32)
        assert bool((scale == s).all()) and codes[0, 0, :16].tolist() == [-7, -6, -6, -4, -4, -2, -2, 0, 0, 2, 2, 4, 4, 6, 6, 7]


@pytest.mark.parametrize("Hq,H,D", [(14, 2, 128), (3, 3, 96), (9, 1, 256)])
def test_every_scale_is_read_and_attended(Hq, H, D):
    """All finite scales there are, of either sign: rows read back exactly, attention within its bounds."""
    g = gen(D)
    c = Cache(g, 3, 700, 16, H, D, I4)
    for t in (c.kb, c.vb):
        b = torch.randint(0, 254, t.shape, generator=g, device="cuda")
        b += b >= 127  # not 0x7F, and not 0xFF: the two NaN
        bits(t)[..., :D // 16] = b[..., :D // 16].to(torch.uint8)
    lens, q = ints([700, 1, 333]), randn(g, 3, Hq, D, dtype=BF16)
    j = torch.arange(333, device="cuda")
    k, v = cp.coverprune_cache_read(c.k, c.v, c.table[2:], ints([0]), starts=ints([0, 333]), tokens=333, **c.kw)
    for what, x in (("k", k), ("v", v)):
        assert torch.equal(wide(x), c.values(what, c.at(2, j)))
    scale = 1e-4 * D ** -0.5
    r = cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, scale=scale, lse=True, **c.kw)
    want, L, _, dout, dlse, _ = attention(q, c, c.table, lens, 0, None, scale)
    assert_stored(r["out"], want, dout, "out")
    assert bool(((r["lse"].double() - L).abs() <= dlse).all())
