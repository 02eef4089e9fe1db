"""Caches of 4 bits, rows read back, the weights of keys added up, and eviction, against their definitions in 64 bits.

Tolerances are bounds on the roundings that the operators state (those of test_gpu_serve.py, and):
  4 bits   a component is within half a step s h of what it stands for, as max |x| / (7 s h) is at most 1 + 2^-4 where
           the scale is a normal number (7 (1 + 2^-4) rounds to 7), and the division adds 8 2^-24 steps
  weight   exp(s - lse) with s off by d and lse off by dlse is off by d + dlse of itself (and 2^-22 for the exponential,
           log 2's factor and the sums: (Hq + 8) 2^-24); added to what was there in one more rounding, 2^-24
"""
import math

import pytest
import torch

import paper_2608_13226_gb300 as cp
from test_gpu_serve import BF16, E4M3, F32, assert_stored, bits, freq, gen, pool, randn, turned, wide

pytestmark = pytest.mark.gpu
I4 = torch.uint8


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_13226_gb300 import build
    build.build()
    cp.load()


def block_bytes(D):
    return (D // 16 + 3) // 4 * 4


class Cache:
    """A paged cache of any type with random contents and what the calls want of it."""

    def __init__(self, g, B, keys, page, H, D, cdt, heads_first=False, scales=False, width=None, shift=0):
        self.W = width or max(1, -(-keys // page))
        self.pages, self.page, self.H, self.D, self.cdt = B * self.W + 2, page, H, D, cdt
        self.table = torch.randperm(self.pages, generator=g, device="cuda")[:B * self.W].reshape(B, self.W).int()

        def shaped(n):
            return (self.pages, H, page, n) if heads_first else (self.pages, page, H, n)

        def put(t):
            return t.permute(0, 2, 1, 3) if heads_first else t

        self.kb = self.vb = None
        if cdt == I4:
            self.k, self.v = (put(torch.randint(1, 16, shaped(D // 2), generator=g, device="cuda", dtype=torch.uint8) +
                                  16 * torch.randint(1, 16, shaped(D // 2), generator=g, device="cuda", dtype=torch.uint8)) for _ in "kv")
            sb = block_bytes(D)
            if shift:  # scales that start on 4 bytes only
                raw = torch.zeros(2, math.prod(shaped(sb + 4)), dtype=torch.uint8, device="cuda").view(E4M3)
                self.kb, self.vb = (put(raw[i].view(shaped(sb + 4))[..., 4:]) for i in (0, 1))
            else:
                self.kb, self.vb = (put(torch.zeros(shaped(sb), dtype=torch.uint8, device="cuda").view(E4M3)) for _ in "kv")
            for t in (self.kb, self.vb):
                x = (0.05 + 0.4 * torch.rand(t.shape, generator=g, device="cuda")).to(E4M3)
                bits(t).copy_(bits(x))
                bits(t)[..., D // 16:] = 0x7F  # padding: NaN
        else:
            self.k, self.v = pool(g, self.pages, page, H, D, cdt, heads_first), pool(g, self.pages, page, H, D, cdt, heads_first)
        self.ks, self.vs = (0.5 + torch.rand(2, H, generator=g, device="cuda")) * (0.02 if cdt == E4M3 else 1.0) if scales else (None, None)

    @property
    def kw(self):
        return dict(k_block=self.kb, v_block=self.vb)

    @property
    def scaled(self):
        return dict(self.kw, k_scale=self.ks, v_scale=self.vs)

    def at(self, b, j):
        return self.table[b].long()[j // self.page], j % self.page

    def values(self, what, at, head=slice(None)):
        """Rows [n, H, D] (or [n, D] of one head) at (pages, slots) in 64 bits."""
        x = bits(self.k if what == "k" else self.v)[:, :, head][at]
        scale = self.ks if what == "k" else self.vs
        if self.cdt == I4:
            n = torch.stack([x & 15, x >> 4], -1).flatten(-2).double() - 8
            s = bits(self.kb if what == "k" else self.vb)[:, :, head][at].view(E4M3).float().double()[..., :self.D // 16]
            x = n * s.repeat_interleave(16, -1)
        else:
            x = wide(x.view(self.cdt))
        if scale is None:
            return x
        return x * (scale.double()[:, None] if isinstance(head, slice) else float(scale[head]))

    def bytes(self):
        """Everything it holds, for comparing."""
        return [bits(t).clone() for t in (self.k, self.v, self.kb, self.vb) if t is not None]


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def flat(new, past):
    """Sequence and key of each of the tokens."""
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
    return seq, torch.cat([torch.arange(p, p + n) for p, n in zip(past, new)]).cuda()


# ------------------------------------------------------------------ append and read
def as_fours(x, head):
    """(codes as whole numbers, scales e4m3) of rows x [T, H, D] float32: the definition, an operation at a time."""
    x = x.unflatten(-1, (-1, 16))
    h = torch.ones(x.shape[1], device=x.device) if head is None else head
    s = (x.abs().amax(-1) / (7.0 * h[:, None])).clamp(max=448.0).to(E4M3)
    step = (s.float() * h[:, None])[..., None]
    return torch.where(step == 0, 0.0, (x / step)).round().clamp(-7, 7).flatten(-2), s


def check_append(seed, new, past, page, Hq, H, D, rot, dtype, heads_first=False, layout="half", scales=False, starts=True, view=0,
                 padding=0, use_pos=True, in_place=False, shift=0):
    g = gen(seed)
    B, T = len(new), sum(new) + padding
    c = Cache(g, B, max(p + n for p, n in zip(past, new)), page, H, D, I4, heads_first, scales, shift=shift)
    before = c.bytes()
    fused = randn(g, T, Hq + 2 * H, D + view, dtype=dtype)[..., view:] * (8 * torch.exp(0.3 * torch.randn(T, 1, 1, generator=g, device="cuda"))).to(dtype)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:]
    q0 = q.clone()
    st = ints([0] + new).cumsum(0).int() if starts else None
    lens, status = ints(past), ints([0])
    pos = torch.randint(0, 100000, (T,), generator=g, device="cuda") if use_pos else None
    f = freq(rot // 2) if rot else None
    r = cp.coverprune_cache_append(k, v, c.k, c.v, c.table, lens, starts=st, pos=pos, inv_freq=f, layout=layout, q=q if Hq else None,
                                   q_out=q if in_place else None, status=status, **c.scaled)
    assert int(status) == 0 and r["lens"].tolist() == [p + n for p, n in zip(past, new)]
    n = T - padding
    seq, slot = flat(new, past)
    at = (c.table.long()[seq, slot // page], slot % page)
    where = slot if pos is None else pos[:n]
    for what, x, head in (("k", k[:n], c.ks), ("v", v[:n], c.vs)):
        cache, blocks = (c.k, c.kb) if what == "k" else (c.v, c.vb)
        want, mag = (turned(x, where, f, layout) if rot else (wide(x), 0 * wide(x))) if what == "k" else (wide(x), 0 * wide(x))
        got = c.values(what, at)
        s = bits(blocks)[at].view(E4M3).float().double()[..., :D // 16]
        h = 1.0 if head is None else head.double()[:, None]
        step = (s * h).repeat_interleave(16, -1)
        top = want.unflatten(-1, (-1, 16)).abs().amax(-1) / (7 * h)
        off = 5e-7 * mag.unflatten(-1, (-1, 16)).amax(-1) / (7 * h)
        assert bool((top > 2.0 ** -6).all())  # scales that are normal numbers
        assert bool(((s - top).abs() <= (2.0 ** -4 + 2.0 ** -22) * top + off).all())
        assert bool(((got - want).abs() <= (0.5 + 2.0 ** -20) * step + 5e-7 * mag).all())
        assert bool((bits(blocks)[at][..., D // 16:] == 0).all())
        if what == "v" or not rot:  # every operation is one of float32: the same numbers
            codes, scale = as_fours(x.float(), head)
            held = bits(cache)[at]
            assert torch.equal(torch.stack([held & 15, held >> 4], -1).flatten(-2).float() - 8, codes)
            assert torch.equal(bits(blocks)[at][..., :D // 16], bits(scale))
    if Hq:
        want, mag = turned(q0[:n], where, f, layout) if rot else (wide(q0[:n]), 0 * wide(q0[:n]))
        assert_stored(r["q"][:n], want, 5e-7 * mag, "queries")
        if in_place:
            assert torch.equal(q[n:], q0[n:])
    for t, t0 in zip((c.k, c.v, c.kb, c.vb), before):  # nothing else was written
        other = torch.ones(t.shape[:2], dtype=torch.bool, device="cuda")
        other[at] = False
        assert torch.equal(bits(t)[other], t0[other])
    check_read(c, lens, st, seq, slot, T)


def check_read(c, lens, st, seq, slot, T):
    """Rows read back are what the cache stands for, rounded once."""
    at, n = (c.table.long()[seq, slot // c.page], slot % c.page), len(seq)
    for dt in {F32: [F32], BF16: [BF16]}.get(c.cdt, [BF16, F32]):
        status = ints([0])
        k, v = cp.coverprune_cache_read(c.k, c.v, c.table, lens, starts=st, tokens=T, dtype=dt, status=status, **c.scaled)
        assert k.shape == v.shape == (T, c.H, c.D) and k.dtype == v.dtype == dt and int(status) == 0
        for what, x in (("k", k[:n]), ("v", v[:n])):
            want = c.values(what, at)
            if (c.ks if what == "k" else c.vs) is None:
                assert torch.equal(wide(x), want)  # exact in either type
            else:
                assert_stored(x, want, 2.0 ** -24 * want.abs(), what)
        wideo = torch.full((T, 2 * c.H, c.D + 3), 7.0, device="cuda", dtype=dt)  # rows of a larger tensor, odd strides
        r = cp.coverprune_cache_read(c.k, c.v, c.table, lens, starts=st, k_out=wideo[:, :c.H, 1:-2], v_out=wideo[:, c.H:, 1:-2], **c.scaled)
        assert torch.equal(r[0][:n], k[:n]) and torch.equal(r[1][:n], v[:n])
        assert bool((wideo[n:] == 7).all()) and bool((wideo[..., 0] == 7).all()) and bool((wideo[..., -2:] == 7).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,rot,layout,page,hf", [(64, 64, "half", 16, False), (128, 128, "interleaved", 7, True), (128, 128, "half", 32, True),
                                                  (96, 40, "half", 1, False), (256, 64, "interleaved", 100, True), (32, 20, "half", 33, False),
                                                  (160, 0, "half", 4, False), (224, 222, "half", 16, False), (96, 96, "interleaved", 16, True),
                                                  (32, 2, "interleaved", 5, False), (256, 256, "half", 16, False)])
def test_append(dtype, D, rot, layout, page, hf):
    check_append(D + page, [5, 0, 1, 63, 0], [0, 9, 40, 3, 0], page, 6, 3, D, rot, dtype, hf, layout, True, padding=4)
    check_append(D + page + 1, [1] * 9, [0, 1, 2, 15, 16, 31, 32, 99, 100], page, 4, 2, D, rot, dtype, hf, layout, starts=False, use_pos=False,
                 in_place=True)
    check_append(D + page + 2, [7, 700], [3, 0], page, 3, 1, D, rot, dtype, hf, layout, view=3, in_place=True, shift=1)


@pytest.mark.parametrize("Hq,H,D,rot", [(28, 4, 128, 128), (0, 1, 64, 0), (5, 5, 96, 48)])
def test_append_many_tokens(Hq, H, D, rot):
    check_append(D + Hq, [9000, 0, 12345, 7001, 1], [3, 0, 100, 0, 77], 16, Hq, H, D, rot, BF16, scales=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,rot", [(96, 24), (32, 8), (64, 40), (128, 72), (128, 6), (96, 30), (256, 248)])
def test_append_turns_parts(dtype, D, rot):
    """Halves that are not vectors of 16 bytes apart, in rows that are (and of a larger tensor)."""
    check_append(D + rot, [5, 0, 300], [0, 9, 40], 7, 6, 3, D, rot, dtype, padding=3)
    check_append(D + rot + 1, [70, 1], [3, 16], 16, 3, 1, D, rot, dtype, True, scales=True, view=8, in_place=True)


def test_append_and_read_many_sequences():
    """More sequences than are counted at once, most of them empty or short, and one among them long."""
    new = [(i * 7 % 5) * (i % 3 == 0) for i in range(900)]
    new[417] = 333
    check_append(1, new, [i % 4 for i in range(900)], 4, 2, 1, 32, 32, BF16, padding=5)
    check_append(2, [0] * 256 + [1] + [0] * 40, [0] * 297, 1, 0, 1, 64, 0, F32)
    check_append(3, [0] * 255 + [2], [3] * 256, 2, 1, 2, 32, 16, BF16)


def test_append_specials():
    """Infinities saturate with their block, a NaN makes its 16 components NaN, what is too small becomes 0."""
    v = torch.randn(1, 1, 96, device="cuda")
    v[..., 3], v[..., 20], v[..., 40] = math.inf, math.nan, -math.inf
    v[..., 48:64], v[..., 64:80] = 0.0, 1e-4 * torch.arange(16, device="cuda")  # 1e-4 * 15 / 7 is below 2^-10
    v[..., 80:] = 0.0
    v[..., 95] = -1e9
    c = Cache(gen(0), 1, 1, 1, 1, 96, I4)
    lens = ints([0])
    cp.coverprune_cache_append(v, v, c.k, c.v, c.table, lens, **c.kw)
    k, x = cp.coverprune_cache_read(c.k, c.v, c.table, lens, dtype=F32, **c.kw)
    assert torch.equal(k.nan_to_num(9e9), x.nan_to_num(9e9))
    x = x[0, 0].tolist()
    assert x[3] == 7 * 448 and x[40] == -7 * 448 and all(y == 0 for i, y in enumerate(x[:16]) if i != 3)
    assert all(math.isnan(y) for y in x[16:32]) and not any(math.isnan(y) for y in x[:16] + x[32:])
    assert x[48:80] == [0.0] * 32 and x[95] == -7 * 448 and x[80:95] == [0.0] * 15
    assert bits(c.kb)[c.table[0, 0].item(), 0, 0, 6:].tolist() == [0, 0]


@pytest.mark.parametrize("cdt", [I4, BF16, F32, E4M3])
@pytest.mark.parametrize("D,page,hf", [(128, 16, False), (64, 7, True), (96, 1, False), (160, 3, True), (16, 4, False), (24, 5, True), (4, 2, False), (256, 64, False)])
def test_read(cdt, D, page, hf):
    if D % {I4: 32, E4M3: 16, BF16: 8, F32: 4}[cdt]:
        pytest.skip("rows of the cache are 16 bytes or a multiple")
    g = gen(D)
    new, past = [5, 0, 300, 1], [0, 4, 17, 2]
    for scales in (False, True):
        c = Cache(g, 4, 320, page, 3, D, cdt, hf, scales)
        st = ints([0] + new).cumsum(0).int()
        check_read(c, ints(past), st, *flat(new, past), sum(new) + 3)
        check_read(c, ints(past), None, *flat([1] * 4, past), 4)


@pytest.mark.parametrize("cdt", [I4, BF16])
def test_rows_that_are_not_there(cdt):
    """Bad pages, a full sequence and a negative length: skipped by the append, read as 0."""
    g = gen(1)
    c = Cache(g, 5, 8, 4, 2, 64, cdt)
    c.table.copy_(ints([[0, 1], [2, c.pages], [3, -1], [4, 5], [0, 1]]))
    lens = ints([8, 4, 5, 7, -2])
    before = c.bytes()
    k = randn(g, 5, 2, 64, dtype=BF16) + 1
    status = ints([0])
    q = randn(g, 5, 3, 64, dtype=BF16)
    r = cp.coverprune_cache_append(k, k, c.k, c.v, c.table, lens, q=q, status=status, **c.kw)
    assert int(status) == cp.CP_EINVAL and r["lens"].tolist() == [8, 5, 6, 8, -2] and torch.equal(r["q"], q)
    for t, t0 in zip((c.k, c.v, c.kb, c.vb), before):
        t0[5, 3] = bits(t)[5, 3]
        assert torch.equal(bits(t), t0)
    status.zero_()
    x, y = cp.coverprune_cache_read(c.k, c.v, c.table, lens, status=status, **c.kw)
    assert int(status) == cp.CP_EINVAL and bool((x[3] != 0).any()) and bool((x[[0, 1, 2, 4]] == 0).all()) and bool((y[[0, 1, 2, 4]] == 0).all())


# ------------------------------------------------------------------ attention
def attention(q, c, table, lens, window, keep, scale, weight=None):
    """(out, lse, weight after the call, bounds on them) in 64 bits, a head of a sequence at a time."""
    B, Hq, D = q.shape
    G = Hq // c.H
    out, lse = torch.zeros(B, Hq, D, dtype=torch.float64, device="cuda"), torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    dout, dlse = torch.zeros_like(out), torch.zeros_like(lse)
    w = dw = None
    if weight is not None:
        w, dw = weight.double(), torch.zeros_like(weight, dtype=torch.float64)
    rounds = {F32: 0.0, BF16: 2.0 ** -8, E4M3: 2.0 ** -11, I4: 2.0 ** -11}[c.cdt]
    for b, n in enumerate(lens.tolist()):
        n = min(max(n, 0), table.shape[1] * c.page)
        j = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        if keep is not None:
            j = j[keep[b][j]]
        pg = table[b].long()[j // c.page]
        j, pg = j[(pg >= 0) & (pg < c.pages)], pg[(pg >= 0) & (pg < c.pages)]
        if not len(j):
            continue
        for h in range(c.H):
            k, v = c.values("k", (pg, j % c.page), h), c.values("v", (pg, j % c.page), h)
            at = slice(h * G, (h + 1) * G)
            qq = wide(q[b, at])
            s = qq @ k.T * scale
            ds = ((D + 4) * 2.0 ** -24 * (qq.abs() @ k.abs().T) * abs(scale)).amax(-1, keepdim=True)
            L = s.logsumexp(-1, keepdim=True)
            p = (s - L).exp()
            out[b, at], lse[b, at] = p @ v, L[:, 0]
            some = 2 * ds + 2 * s.abs().amax(-1, keepdim=True) * 2.0 ** -23 + (len(j) + 16) * 2.0 ** -24
            dout[b, at] = (rounds + some) * (p @ v.abs())
            if c.cdt in (E4M3, I4):
                dout[b, at] += len(j) * 2.0 ** -25 * v.abs().amax() * (s.amax(-1, keepdim=True) - L).exp()
            dlse[b, at] = (some + 2.0 ** -22 * (1 + L.abs()))[:, 0]
            if w is not None:
                w[b, j] += p.sum(0)
                off = ds + dlse[b, at][:, None] + (s.abs() + L.abs()) * 2.0 ** -22 + (Hq + 8) * 2.0 ** -24
                dw[b, j] += (p * off).sum(0)
    if w is not None:
        dw += 2.0 ** -23 * w.abs()
    return out, lse, w, dout, dlse, dw


def check_decode(seed, lens, page, Hq, H, D, cdt, window=0, keep=None, heads_first=False, scales=False, junk=False, width=None, sharp=1.0,
                 scale=None, q_view=False, weigh=False, shift=0):
    g = gen(seed)
    B, dt = len(lens), F32 if cdt == F32 else BF16
    c = Cache(g, B, max(max(lens), 1), page, H, D, cdt, heads_first, scales, width, shift)
    keys = c.W * page
    kp = torch.rand(B, keys + 3, generator=g, device="cuda")[:, :keys] < keep if keep is not None else None
    if junk:  # whatever is not visible holds NaN
        j, n = torch.arange(keys, device="cuda")[None], torch.tensor(lens, device="cuda")[:, None]
        vis = (j < n) & (j >= n - (window or 1 << 40))
        vis = vis & kp if kp is not None else vis
        mark = torch.ones(c.pages, page, dtype=torch.bool, device="cuda")
        seq = torch.arange(B, device="cuda")[:, None].expand_as(vis)
        mark[c.table.long()[seq, j.expand_as(vis) // page][vis], (j.expand_as(vis) % page)[vis]] = False
        for t in (c.kb, c.vb) if cdt == I4 else (c.k, c.v):
            bits(t)[mark] = bits(torch.full((1,), math.nan, device="cuda").to(t.dtype))[0]
    q = (randn(g, B, Hq + 2, D + 8) * sharp).to(dt)[:, 1:Hq + 1, 3:D + 3] if q_view else (randn(g, B, Hq, D) * sharp).to(dt)
    lt = ints(lens)
    tb = torch.where(torch.arange(c.W, device="cuda")[None] * page < lt[:, None], c.table, -1)
    w = torch.rand(B, keys + 5, generator=g, device="cuda")[:, :keys + 2] if weigh else None
    w0 = w.clone() if weigh else None
    status = ints([0])
    kw = dict(window=window, keep=kp, lse=True, scale=scale, status=status, **c.scaled)
    r = cp.coverprune_decode_attention(q, c.k, c.v, tb, lt, weight=w, **kw)
    want, L, ww, dout, dlse, dw = attention(q, c, tb, lt, window, kp, D ** -0.5 if scale is None else scale, w0)
    assert int(status) == 0
    assert_stored(r["out"], want, dout, "out")
    got, fine = r["lse"].double(), L > -math.inf
    assert torch.equal(got == -math.inf, ~fine)
    assert bool(((got - L).abs()[fine] <= dlse[fine]).all()), f"lse off by {(got - L).abs()[fine].max()}"
    assert bool((r["out"][~fine] == 0).all())
    if weigh:
        assert bool(((w.double() - ww).abs() <= dw).all()), f"weights: {((w.double() - ww).abs() - dw).max()} over"
        assert torch.equal(w[ww == w0.double()], w0[ww == w0.double()])  # of keys that are not visible
        # the call without weights is a program of its own, whose products and sums may be contracted
        # elsewhere: the same bounds, not the same bits
        plain = cp.coverprune_decode_attention(q, c.k, c.v, tb, lt, **kw)
        assert_stored(plain["out"], want, dout, "out without weights")
        assert bool(((plain["lse"].double() - L).abs()[fine] <= dlse[fine]).all())
    v = w0.clone() if weigh else None
    again = cp.coverprune_decode_attention(q, c.k, c.v, tb, lt, weight=v, ws=r["ws"], **{**kw, "lse": False})
    assert torch.equal(bits(again["out"]), bits(r["out"])) and (not weigh or torch.equal(v, w))
    return r


HEADS = [(1, 1, 64), (28, 4, 128), (8, 8, 128), (16, 2, 96), (9, 1, 256), (24, 2, 160), (33, 3, 64), (40, 2, 128), (64, 1, 32), (34, 2, 256),
         (14, 2, 224), (10, 5, 192)]


@pytest.mark.parametrize("Hq,H,D", HEADS)
@pytest.mark.parametrize("scales", [False, True])
def test_fours_heads(Hq, H, D, scales):
    check_decode(Hq * D, [0, 1, 15, 16, 17, 31, 32, 33, 130, 1000], 16, Hq, H, D, I4, scales=scales, shift=scales)


@pytest.mark.parametrize("page", [1, 3, 16, 64, 100, 1024])
@pytest.mark.parametrize("hf", [False, True])
def test_fours_pages(page, hf):
    check_decode(page, [63, 64, 65, 255, 256, 257, 2, 700], page, 14, 2, 128, I4, heads_first=hf, scales=True, junk=True)
    check_decode(page, [63, 64, 65, 255, 256, 257, 2, 700], page, 6, 2, 96, I4, heads_first=hf, junk=True, q_view=True)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 500, 5000])
def test_fours_window(window):
    check_decode(window, [0, 1, 64, 65, 449, 2000], 16, 8, 2, 64, I4, window=window, scales=True, junk=True)


@pytest.mark.parametrize("keep,window", [(0.0, 0), (0.02, 0), (0.15, 0), (0.5, 300), (0.97, 0), (1.0, 0)])
def test_fours_keep(keep, window):
    check_decode(int(100 * keep), [1500, 700, 64, 3, 0], 16, 14, 2, 128, I4, window=window, keep=keep, junk=True)
    check_decode(int(100 * keep), [300] * 40, 16, 8, 8, 64, I4, window=window, keep=keep, junk=True)


@pytest.mark.parametrize("lens,Hq,H,D,page", [([20000, 3, 0, 9999], 14, 2, 128, 16), ([300] * 700, 7, 1, 64, 7), ([100, 20, 300, 4] * 100, 28, 4, 128, 16),
                                              ([70001], 32, 8, 128, 64), ([5, 900] * 40, 12, 1, 256, 100), ([17, 32], 6, 3, 96, 8),
                                              ([2500] * 33, 20, 20, 64, 16)])
def test_fours_lengths(lens, Hq, H, D, page):
    """By warps, blocks, clusters and one line, exact and wide tables."""
    check_decode(len(lens), lens, page, Hq, H, D, I4, scales=True)
    check_decode(len(lens), lens, page, Hq, H, D, I4, width=-(-max(lens) * 3 // page) + 5, weigh=True)


@pytest.mark.parametrize("sharp,scale", [(30.0, None), (0.001, 5.0), (1.0, -0.3), (8.0, 0.0)])
def test_fours_sharp_and_scaled(sharp, scale):
    check_decode(3, [0, 70, 900, 2500], 16, 14, 2, 128, I4, sharp=sharp, scale=scale, scales=True, weigh=True)


def test_fours_nan_scale_shows():
    """A visible scale that is NaN reaches the outputs of its block, or as a key's every one; other sequences are as they were."""
    c = Cache(gen(2), 3, 200, 16, 2, 128, I4)
    q, lens = randn(gen(3), 3, 4, 128, dtype=BF16), ints([200, 150, 20])
    good = cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, lse=True, **c.kw)
    bits(c.vb)[c.table[0, 3].item(), 5, 1, 2] = 0x7F
    bits(c.kb)[c.table[1, 0].item(), 0, 0, 7] = 0x7F
    r = cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, lse=True, **c.kw)
    nan = r["out"].isnan()
    assert torch.equal(r["out"][2], good["out"][2])
    assert bool(nan[0, 2:, 32:48].all()) and int(nan[0].sum()) == 2 * 16 and torch.equal(r["out"][0][~nan[0]], good["out"][0][~nan[0]])
    assert bool(nan[1, :2].all()) and bool(r["lse"][1, :2].isnan().all()) and torch.equal(r["out"][1, 2:], good["out"][1, 2:])


# ------------------------------------------------------------------ weights
TYPES = [(BF16, False), (F32, False), (E4M3, True), (I4, True)]


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("Hq,H,D", [(1, 1, 64), (28, 4, 128), (2, 2, 128), (9, 1, 256), (33, 3, 64), (40, 2, 128), (64, 1, 32), (100, 4, 96)])
def test_weights_heads(Hq, H, D, cdt, scales):
    check_decode(Hq + D, [0, 1, 15, 16, 17, 33, 130, 1000], 16, Hq, H, D, cdt, scales=scales, weigh=True, junk=True)


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("keep,window", [(None, 1), (None, 100), (0.0, 0), (0.1, 0), (0.5, 300), (0.9, 7)])
def test_weights_visible(keep, window, cdt, scales):
    check_decode(window, [1500, 700, 64, 3, 0, 4000], 16, 14, 2, 128, cdt, window=window, keep=keep, scales=scales, weigh=True, junk=True)
    check_decode(window, [200] * 700, 7, 5, 1, 64, cdt, window=window, keep=keep, scales=scales, weigh=True, junk=True)


@pytest.mark.parametrize("cdt,scales", TYPES)
def test_weights_ways(cdt, scales):
    """Keys dealt out by one line, clusters, blocks and warps."""
    for lens, Hq, H, D in (([8000, 30, 12000], 14, 2, 128), ([700], 7, 1, 64), ([250, 100] * 20, 6, 2, 128), ([100] * 900, 4, 1, 64), ([12], 8, 8, 64),
                           ([3000, 100] * 60, 16, 2, 128)):
        check_decode(len(lens), lens, 16, Hq, H, D, cdt, scales=scales, weigh=True)


@pytest.mark.parametrize("cdt", [BF16, F32, E4M3, I4])
def test_weights_bad_pages_and_nan(cdt):
    """Keys on bad pages get nothing, lengths out of range are cut; a NaN makes its sequence's weights NaN, of visible keys only."""
    g = gen(7)
    c = Cache(g, 4, 64, 16, 2, 64, cdt)
    q = randn(g, 4, 6, 64, dtype=F32 if cdt == F32 else BF16)
    lens, status = ints([64, 100, -3, 40]), ints([0])
    c.table[0, 1], c.table[1, 2] = -1, c.pages
    w = torch.zeros(4, 70, device="cuda")
    w[:] = 1.0
    r = cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, weight=w, status=status, lse=True, **c.kw)
    _, L, want, _, dlse, dw = attention(q, c, c.table, lens, 0, None, 0.125, torch.ones(4, 70, device="cuda"))
    assert int(status) == cp.CP_EINVAL and bool(((w.double() - want).abs() <= dw).all())
    assert bool((w[0, 16:32] == 1).all()) and bool((w[1, 32:48] == 1).all()) and bool((w[2] == 1).all()) and bool((w[:, 64:] == 1).all())
    q[3, 0, 0] = math.nan
    cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, weight=w, ws=r["ws"], **c.kw)
    assert bool(w[3, :40].isnan().all()) and bool((w[3, 40:] == 1).all()) and not bool(w[:3].isnan().any())


def test_weights_sum_to_heads():
    """Over the keys of a sequence a call adds 1 a query head."""
    c = Cache(gen(0), 3, 5000, 16, 4, 128, I4, scales=True)
    w, ws = torch.zeros(3, c.W * 16, device="cuda"), None
    for i in range(3):
        r = cp.coverprune_decode_attention(randn(gen(i), 3, 28, 128, dtype=BF16), c.k, c.v, c.table, ints([5000, 1, 333]), weight=w, ws=ws, **c.scaled)
        ws = r["ws"]
    assert bool(((w.double().sum(1) - 84).abs() <= 84 * 5100 * 2.0 ** -24).all())


# ------------------------------------------------------------------ eviction
def chosen(weight, n, left, first, recent):
    """The keys that stay, as a list: sorted by (NaN lowest) weight, the earlier of equals first."""
    if n <= left:
        return list(range(n))
    mid = range(first, n - recent)
    def rank(j):
        x = weight[j]
        return (1, 0.0, j) if x != x else (0, -x, j)
    best = sorted(mid, key=rank)[:left - first - recent]
    return list(range(first)) + sorted(best) + list(range(n - recent, n))


def check_evict(seed, lens, left, first, recent, page, H, D, cdt, heads_first=False, weights=None, width=None, ties=False):
    g = gen(seed)
    B = len(lens)
    c = Cache(g, B, max(max(lens), 1), page, H, D, cdt, heads_first, width=width)
    keys = c.W * page
    w = torch.exp(3 * torch.randn(B, keys + 4, generator=g, device="cuda"))[:, :keys + 3]
    if ties:
        w = (w * 3).floor() / 3
    if weights is not None:
        w[:, :len(weights)] = torch.tensor(weights, device="cuda")
    before, w0, status = c.bytes(), w.clone(), ints([0])
    r = cp.coverprune_cache_evict(c.k, c.v, c.table, ints(lens), w, left, first=first, recent=recent, status=status, **c.kw)
    assert int(status) == 0 and torch.equal(w.nan_to_num(-7.0), w0.nan_to_num(-7.0))
    assert r["kept"].shape == (B, left) and r["weight"].shape == w.shape
    host = w.tolist()
    for b, n in enumerate(lens):
        n = min(max(n, 0), keys)
        stay = chosen(host[b], n, left, first, recent)
        m = len(stay)
        assert r["lens"][b].item() == (lens[b] if lens[b] < 0 else m)
        assert r["kept"][b].tolist() == stay + [-1] * (left - m)
        assert torch.equal(bits(r["weight"][b, :m]), bits(w[b, stay])) and bool((r["weight"][b, m:] == 0).all())
        j = torch.tensor(stay, device="cuda", dtype=torch.long)
        to, of = c.at(b, torch.arange(m, device="cuda")), c.at(b, j)
        moved = [t.clone() for t in before]
        for t, t0 in zip(moved, before):
            t[to] = t0[of]
        before = moved
    for t, want in zip((c.k, c.v, c.kb, c.vb), before):
        assert torch.equal(bits(t), want)
    return c, r


@pytest.mark.parametrize("cdt", [BF16, F32, E4M3, I4])
@pytest.mark.parametrize("D,H,page,hf", [(128, 4, 16, False), (64, 3, 7, True), (96, 1, 1, False), (32, 2, 100, True), (256, 2, 64, False), (224, 1, 5, False)])
def test_evict(cdt, D, H, page, hf):
    check_evict(D, [0, 1, 299, 300, 301, 400, 1000, 302], 300, 4, 16, page, H, D, cdt, hf)


@pytest.mark.parametrize("D,H,cdt", [(80, 3, BF16), (16, 2, E4M3), (8, 1, BF16), (4, 1, F32), (80, 2, F32)])
def test_evict_narrow_rows(D, H, cdt):
    check_evict(D, [700, 65, 64, 63], 64, 0, 5, 16, H, D, cdt)


@pytest.mark.parametrize("D,H,cdt,hf", [(96, 2, BF16, False), (80, 1, BF16, True), (256, 1, F32, False), (128, 4, I4, False), (64, 4, I4, True), (48, 3, E4M3, False)])
@pytest.mark.parametrize("B,cut", [(21, [20]), (33, [0, 31, 32]), (256, [7, 255]), (257, [3, 256]), (300, [])])
def test_evict_few_of_many(B, cut, D, H, cdt, hf):
    """Sequences that are cut between many that are not: blocks of those help."""
    lens = [(7 * b) % 600 + 1 for b in range(B)]
    for i, b in enumerate(cut):
        lens[b] = 640 + 37 * i
    check_evict(B + D, lens, 600, 2, 50, 16, H, D, cdt, hf)


@pytest.mark.parametrize("left,first,recent", [(0, 0, 0), (1, 0, 0), (1, 1, 0), (1, 0, 1), (50, 25, 25), (50, 0, 50), (50, 50, 0), (50, 0, 0), (999, 10, 10),
                                               (1000, 0, 0), (5000, 7, 9)])
def test_evict_budgets(left, first, recent):
    check_evict(left, [1000, 51, 50, 2, 0, 998], left, first, recent, 16, 2, 64, BF16)
    check_evict(left, [1000, 51, 50, 2, 0, 998], left, first, recent, 16, 2, 64, I4, ties=True)


def test_evict_ties_and_specials():
    """The earlier of equal weights stays; NaN is less than -infinity, -0 equals 0."""
    inf, nan = math.inf, math.nan
    check_evict(0, [20], 9, 0, 0, 4, 1, 64, BF16, weights=[0.0, -0.0, nan, 1.0, -inf, inf, -1.0, 0.0, -0.0, 1e-45, -1e-45, nan, inf, 2.0, 2.0, nan, -inf, 0.0, 3e38, -3e38])
    check_evict(0, [20], 17, 0, 0, 4, 1, 64, BF16, weights=[nan] * 3 + [-inf] * 3 + [0.0, -0.0] * 7)
    check_evict(0, [20], 18, 1, 1, 4, 1, 64, BF16, weights=[nan] * 20)
    check_evict(0, [1000, 800], 333, 3, 3, 16, 1, 64, F32, weights=[0.25] * 1000)
    check_evict(0, [1000, 800], 333, 3, 3, 16, 1, 64, F32, ties=True)
    check_evict(0, [5000] * 3, 2500, 0, 0, 16, 1, 64, BF16, weights=[1.0 + 2.0 ** -23 * (i % 3) for i in range(5000)])


@pytest.mark.parametrize("lens,left,page,D,H,cdt", [([50000, 30, 40001], 20000, 64, 64, 1, BF16), ([200001], 100000, 64, 32, 1, I4),
                                                    ([9000] * 9, 1229, 16, 128, 4, BF16), ([1240] * 64, 1229, 32, 128, 2, E4M3),
                                                    ([140000, 139999], 139000, 100, 8, 1, BF16), ([300001], 123456, 64, 8, 1, BF16),
                                                    ([4000] * 3 + [90] * 160, 77, 7, 8, 1, BF16)])
def test_evict_long(lens, left, page, D, H, cdt):
    """Blocks alone and clusters of them; many turns."""
    check_evict(left, lens, left, 4, 64, page, H, D, cdt, ties=True)


def test_evict_lengths_out_of_range_and_wide_tables():
    check_evict(5, [-3, 500, 64], 60, 2, 3, 16, 2, 64, BF16)
    c, r = check_evict(6, [70, 3], 40, 0, 0, 16, 2, 64, I4, width=3000)
    # rows of 40,000 keys of more sequences than share the device by clusters: weights are read again, not held
    check_evict(7, [700, 3, 120] * 60, 100, 1, 2, 16, 1, 64, BF16, width=2500, ties=True)
    g = gen(3)  # a length beyond the table's row is what the row holds
    c = Cache(g, 1, 32, 16, 1, 64, BF16)
    w = torch.rand(1, 32, generator=g, device="cuda")
    r = cp.coverprune_cache_evict(c.k, c.v, c.table, ints([999]), w, 10, recent=2)
    assert r["lens"].tolist() == [10] and r["kept"][0].tolist() == chosen(w[0].tolist(), 32, 10, 0, 2)


def test_evict_bad_pages():
    """A key that is on a bad page or would come to one is not moved; the others are."""
    c = Cache(gen(4), 2, 64, 16, 2, 64, BF16)
    c.table[0, 2] = -1
    c.table[1, 0] = c.pages + 5
    before = c.bytes()
    w = torch.arange(64.0, device="cuda").repeat(2, 1)
    status = ints([0])
    r = cp.coverprune_cache_evict(c.k, c.v, c.table, ints([64, 64]), w, 30, status=status)
    assert int(status) == cp.CP_EINVAL and r["kept"].tolist() == [list(range(34, 64))] * 2
    for t, t0 in zip((c.k, c.v), before):
        want = t0.clone()
        for b in range(2):
            for i in range(30):
                p, q = int(c.table[b, (34 + i) // 16]), int(c.table[b, i // 16])
                if 0 <= p < c.pages and 0 <= q < c.pages:
                    want[q, i % 16] = t0[p, (34 + i) % 16]
        assert torch.equal(bits(t), want)


def test_attention_after_eviction():
    """What attention gives on the kept keys is what marks on the whole cache give."""
    for cdt in (BF16, I4):
        c = Cache(gen(9), 3, 900, 16, 2, 128, cdt)
        q, lens = randn(gen(1), 3, 14, 128, dtype=BF16), ints([900, 700, 40])
        w = torch.zeros(3, c.W * 16, device="cuda")
        cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, weight=w, **c.kw)
        # keep marks of the same keys, before the rows move
        marks = torch.zeros(3, c.W * 16, dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens.tolist()):
            marks[b, chosen(w[b].tolist(), n, 100, 2, 10)] = True
        want, L, _, dout, dlse, _ = attention(q, c, c.table, lens, 0, marks, 128 ** -0.5)
        r = cp.coverprune_cache_evict(c.k, c.v, c.table, lens, w, 100, first=2, recent=10, **c.kw)
        assert r["lens"].tolist() == [100, 100, 40]
        got = cp.coverprune_decode_attention(q, c.k, c.v, c.table, r["lens"], lse=True, **c.kw)
        assert_stored(got["out"], want, dout, "out")
        assert bool(((got["lse"].double() - L).abs() <= dlse).all())


# ------------------------------------------------------------------ as they are used
@pytest.mark.parametrize("cdt", [BF16, I4])
def test_graph_of_steps(cdt):
    """Append, attention with weights and eviction captured together and replayed: as the same calls made one by one."""
    def make():
        g = gen(11)
        c = Cache(g, 4, 256, 16, 2, 128, cdt)
        return c, ints([200, 130, 5, 128]), torch.rand(4, 256, generator=g, device="cuda")

    g = gen(12)
    x = randn(g, 4, 14 + 4, 128, dtype=BF16)
    at = torch.tensor([900, 800, 700, 600], device="cuda")

    def step(c, lens, w, out, pos):
        r = cp.coverprune_cache_append(x[:, 14:16], x[:, 16:], c.k, c.v, c.table, lens, pos=pos, inv_freq=freq_, q=x[:, :14], **c.kw)
        cp.coverprune_decode_attention(r["q"], c.k, c.v, c.table, r["lens"], weight=w, out=out, **c.kw)
        e = cp.coverprune_cache_evict(c.k, c.v, c.table, r["lens"], w, 128, first=2, recent=8, **c.kw)
        lens.copy_(e["lens"])
        w.copy_(e["weight"])
        pos += 1

    freq_ = freq(64)
    one = make()
    out1, p1 = torch.zeros(4, 14, 128, dtype=BF16, device="cuda"), at.clone()
    for _ in range(4):
        step(*one, out1, p1)
    two = make()
    out2, p2 = torch.zeros_like(out1), at.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*two, out2, p2)  # the first call is not captured
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*two, out2, p2)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out1, out2) and torch.equal(one[1], two[1]) and torch.equal(one[2], two[2])
    assert all(torch.equal(a, b) for a, b in zip(one[0].bytes(), two[0].bytes()))
    assert one[1].tolist() == [128, 128, 9, 128]


def test_streams_side_by_side():
    """The same calls on two streams at once, a workspace each."""
    jobs = []
    for i in range(2):
        c = Cache(gen(i), 8, 3000, 16, 4, 128, I4)
        jobs.append((c, randn(gen(i), 8, 28, 128, dtype=BF16), ints([3000] * 8), torch.zeros(8, c.W * 16, device="cuda")))
    alone = []
    for c, q, lens, _ in jobs:
        w = torch.zeros(8, c.W * 16, device="cuda")
        for _ in range(10):
            r = cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, weight=w, **c.kw)
        alone.append((r["out"], w))
    torch.cuda.synchronize()
    streams, outs, ws = [torch.cuda.Stream() for _ in jobs], [None, None], [None, None]
    for _ in range(10):
        for i, (s, (c, q, lens, w)) in enumerate(zip(streams, jobs)):
            with torch.cuda.stream(s):
                r = cp.coverprune_decode_attention(q, c.k, c.v, c.table, lens, weight=w, ws=ws[i], **c.kw)
                outs[i], ws[i] = r["out"], r["ws"]
    torch.cuda.synchronize()
    for (out, w), got, job in zip(alone, outs, jobs):
        assert torch.equal(out, got) and torch.equal(w, job[3])


def test_autograd_and_versions():
    """Tensors that require a gradient are refused while autograd records; what is written gets a new version."""
    c = Cache(gen(0), 2, 32, 16, 1, 64, I4)
    x, lens, w = randn(gen(1), 2, 1, 64, dtype=BF16), ints([3, 4]), torch.ones(2, 32, device="cuda")
    y = x.clone().requires_grad_()
    for f in (lambda: cp.coverprune_cache_append(y, x, c.k, c.v, c.table, lens, **c.kw),
              lambda: cp.coverprune_decode_attention(y, c.k, c.v, c.table, lens, **c.kw),
              lambda: cp.coverprune_decode_attention(x, c.k, c.v, c.table, lens, weight=w.clone().requires_grad_(), **c.kw),
              lambda: cp.coverprune_cache_evict(c.k, c.v, c.table, lens, w.clone().requires_grad_(), 2, **c.kw)):
        with pytest.raises(ValueError, match="requires a gradient"):
            f()
    with torch.no_grad():
        cp.coverprune_decode_attention(y, c.k, c.v, c.table, lens, **c.kw)

    def bumped(f, *ts):
        v = [t._version for t in ts]
        f()
        assert all(t._version > u for t, u in zip(ts, v))

    bumped(lambda: cp.coverprune_cache_append(x, x, c.k, c.v, c.table, lens, **c.kw), c.k, c.v, c.kb, c.vb)
    bumped(lambda: cp.coverprune_decode_attention(x, c.k, c.v, c.table, lens, weight=w, **c.kw), w)
    nl, nw, kp = ints([0, 0]), torch.empty_like(w), torch.empty(2, 2, dtype=torch.int32, device="cuda")
    bumped(lambda: cp.coverprune_cache_evict(c.k, c.v, c.table, lens, w, 2, new_lens=nl, new_weight=nw, kept=kp, **c.kw), c.k, c.kb, nl, nw, kp)
    k, v = torch.empty_like(x), torch.empty_like(x)
    bumped(lambda: cp.coverprune_cache_read(c.k, c.v, c.table, lens, k_out=k, v_out=v, **c.kw), k, v)


def test_no_tokens_or_sequences():
    c = Cache(gen(0), 2, 32, 16, 1, 64, I4)
    none = torch.zeros(0, 1, 64, device="cuda", dtype=BF16)
    empty, table = ints([]), c.table[:0]
    before = c.bytes()
    assert cp.coverprune_cache_append(none, none, c.k, c.v, table, empty, **c.kw)["lens"].shape == (0,)
    assert cp.coverprune_cache_append(none, none, c.k, c.v, c.table, ints([1, 2]), starts=ints([0, 0, 0]), **c.kw)["lens"].tolist() == [1, 2]
    assert cp.coverprune_cache_read(c.k, c.v, table, empty, **c.kw)[0].shape == (0, 1, 64)
    assert cp.coverprune_cache_read(c.k, c.v, c.table, ints([1, 2]), starts=ints([0, 0, 0]), tokens=0, **c.kw)[1].shape == (0, 1, 64)
    w = torch.zeros(0, 32, device="cuda")
    assert cp.coverprune_decode_attention(none, c.k, c.v, table, empty, weight=w, **c.kw)["out"].shape == (0, 1, 64)
    assert cp.coverprune_cache_evict(c.k, c.v, table, empty, w, 5, **c.kw)["kept"].shape == (0, 5)
    nothing = torch.zeros(2, 0, dtype=torch.int32, device="cuda")
    w = torch.zeros(2, 0, device="cuda")
    r = cp.coverprune_decode_attention(torch.cat([none, torch.ones(2, 1, 64, device="cuda", dtype=BF16)]), c.k, c.v, nothing, ints([4, 0]), weight=w, lse=True, **c.kw)
    assert bool((r["out"] == 0).all()) and bool((r["lse"] == -math.inf).all())
    r = cp.coverprune_cache_evict(c.k, c.v, nothing, ints([4, 0]), w, 3, **c.kw)
    assert r["lens"].tolist() == [0, 0] and r["kept"].tolist() == [[-1] * 3] * 2
    assert all(torch.equal(a, b) for a, b in zip(c.bytes(), before))


def test_refuses_on_gpu():
    c = Cache(gen(0), 2, 32, 16, 2, 64, I4)
    b = Cache(gen(0), 2, 32, 16, 2, 64, BF16)
    x, lens, w = randn(gen(1), 2, 2, 64, dtype=BF16), ints([3, 4]), torch.ones(2, 32, device="cuda")
    cut = dict(k_block=c.kb[..., :2], v_block=c.vb[..., :2])
    other = dict(k_block=c.kb, v_block=c.vb.transpose(1, 2).contiguous().transpose(1, 2))
    for kw in ({}, dict(k_block=c.kb), dict(v_block=c.vb)):
        with pytest.raises(TypeError):
            cp.coverprune_cache_append(x, x, c.k, c.v, c.table, lens, **kw)
    for kw in (cut, other):
        with pytest.raises(ValueError):
            cp.coverprune_decode_attention(x, c.k, c.v, c.table, lens, **kw)
    with pytest.raises(TypeError):
        cp.coverprune_decode_attention(x, c.k, c.v, c.table, lens, k_block=bits(c.kb), v_block=bits(c.vb))
    with pytest.raises(ValueError):  # scales beside a cache that has none
        cp.coverprune_decode_attention(x, b.k, b.v, b.table, lens, **c.kw)
    with pytest.raises(cp.CoverPruneError) as e:
        cp.coverprune_decode_attention(x.float(), c.k, c.v, c.table, lens, **c.kw)
    assert e.value.status == cp.CP_EUNSUPPORTED
    for bad in (w[:, :31], w[:1], w.double(), w.cpu(), w[:1].expand(2, 32), w.t().contiguous().t()):
        with pytest.raises((ValueError, TypeError)):
            cp.coverprune_decode_attention(x, c.k, c.v, c.table, lens, weight=bad, **c.kw)
    for bad in (w[:, :31], w[:1], w.double(), w.cpu(), w.t().contiguous().t()):
        with pytest.raises((ValueError, TypeError)):
            cp.coverprune_cache_evict(c.k, c.v, c.table, lens, bad, 5, **c.kw)
    small = cp.coverprune_decode_attention(x, c.k, c.v, c.table, lens, **c.kw)["ws"]
    with pytest.raises(cp.CoverPruneError) as e:  # the workspace of a call without weights
        cp.coverprune_decode_attention(x, c.k, c.v, c.table, lens, weight=w, ws=small, **c.kw)
    assert e.value.status == cp.CP_EWORKSPACE
    for kw in (dict(left=-1), dict(left=4, first=5), dict(left=4, recent=5), dict(left=4, first=2, recent=3), dict(left=4, first=-1)):
        with pytest.raises(ValueError):
            cp.coverprune_cache_evict(c.k, c.v, c.table, lens, w, **kw, **c.kw)
    for kw in (dict(new_lens=lens), dict(new_weight=w), dict(kept=lens.view(2, 1))):
        with pytest.raises(cp.CoverPruneError) as e:
            cp.coverprune_cache_evict(c.k, c.v, c.table, lens, w, 1, **kw, **c.kw)
        assert e.value.status == cp.CP_EINVAL
    for kw in (dict(new_weight=torch.empty(2, 40, device="cuda")), dict(kept=torch.empty(2, 3, dtype=torch.int32, device="cuda")),
               dict(new_lens=lens.long())):
        with pytest.raises((ValueError, TypeError)):
            cp.coverprune_cache_evict(c.k, c.v, c.table, lens, w, 2, **kw, **c.kw)
    for kw in (dict(tokens=3), dict(tokens=-1), dict(starts=ints([0, 1, 2])), dict(dtype=torch.float16), dict(k_out=x[:, :1]), dict(k_out=x, dtype=F32),
               dict(k_out=x[:1].expand(2, 2, 64))):
        with pytest.raises((ValueError, TypeError)):
            cp.coverprune_cache_read(c.k, c.v, c.table, lens, **kw, **c.kw)
    for cache, dt in ((b, F32), (Cache(gen(0), 2, 32, 16, 2, 64, F32), BF16)):
        with pytest.raises(cp.CoverPruneError) as e:
            cp.coverprune_cache_read(cache.k, cache.v, cache.table, lens, dtype=dt)
        assert e.value.status == cp.CP_EUNSUPPORTED
    with pytest.raises(cp.CoverPruneError) as e:  # rows of 4 bits fill 16 bytes
        n = torch.zeros(4, 16, 1, 24, dtype=torch.uint8, device="cuda")
        cp.coverprune_cache_append(randn(gen(0), 2, 1, 48), randn(gen(0), 2, 1, 48), n, n.clone(), c.table[:, :1] * 0, lens,
                                   k_block=torch.zeros(4, 16, 1, 4, device="cuda").to(E4M3), v_block=torch.zeros(4, 16, 1, 4, device="cuda").to(E4M3))
    assert e.value.status == cp.CP_EUNSUPPORTED


def test_offsets_past_32_bits():
    """Pages more than 2^32 bytes apart, of codes and of scales; scores and weights beyond 2^31 entries."""
    page, H, D, n = 16, 1, 128, 3
    far = (1 << 32) + 64  # bytes from page to page
    raw = torch.zeros(2, 2 * far + page * 64, dtype=torch.uint8, device="cuda")
    rawb = torch.zeros(2, 2 * far + page * 8, dtype=torch.uint8, device="cuda")
    k, v = (r.as_strided((n, page, H, D // 2), (far, 64, 64, 1)) for r in raw)
    kb, vb = (r.as_strided((n, page, H, 8), (far, 8, 8, 1)).view(E4M3) for r in rawb)
    del raw, rawb
    c = Cache(gen(0), 1, 48, page, H, D, I4)
    c.k, c.v, c.kb, c.vb, c.pages = k, v, kb, vb, n
    c.table = ints([[2, 0, 1]])
    x = randn(gen(2), 48, 3, D, dtype=BF16)
    lens, st = ints([0]), ints([0, 48])
    new = cp.coverprune_cache_append(x[:, :1], x[:, 1:2], k, v, c.table, lens, starts=st, **c.kw)["lens"]
    q = x[:1, 2:].contiguous()
    r = cp.coverprune_decode_attention(q, k, v, c.table, new, lse=True, **c.kw)
    want, L, _, dout, dlse, _ = attention(q, c, c.table, new, 0, None, D ** -0.5)
    assert_stored(r["out"], want, dout, "out")
    codes, scale = as_fours(x[:, 1:2].float(), None)
    back = cp.coverprune_cache_read(k, v, c.table, lens, starts=st, tokens=48, **c.kw)[1]
    assert torch.equal(back.float(), codes * scale.float().repeat_interleave(16, -1))
    w = torch.rand(1, 48, device="cuda")
    e = cp.coverprune_cache_evict(k, v, c.table, new, w, 20, **c.kw)
    got = cp.coverprune_cache_read(k, v, c.table, lens, starts=ints([0, 20]), tokens=20, **c.kw)[1]
    assert torch.equal(got, back[e["kept"][0].long()])


def test_scores_past_32_bits():
    """A workspace of scores whose entries pass 2^31: the last sequences' weights are right."""
    B, Hq, W, page = 40, 64, 1 << 16, 16  # 40 * 64 * 2^20 scores, of which few are written
    c = Cache(gen(0), B, 100, page, 1, 64, BF16)
    table = torch.full((B, W), -1, dtype=torch.int32, device="cuda")
    table[:, :c.W] = c.table
    lens = ints([100] * B)
    q = randn(gen(1), B, Hq, 64, dtype=BF16)
    w = torch.zeros(B, W * page, device="cuda")
    cp.coverprune_decode_attention(q, c.k, c.v, table, lens, weight=w)
    for b in (0, B - 1):
        one = torch.zeros(1, c.W * page, device="cuda")
        cp.coverprune_decode_attention(q[b:b + 1], c.k, c.v, c.table[b:b + 1], lens[b:b + 1], weight=one)
        off = (w[b, :c.W * page] - one[0]).abs()
        assert bool((off <= 64 * 2.0 ** -20 * one[0] + 1e-30).all()) and bool((w[b, c.W * page:] == 0).all())
