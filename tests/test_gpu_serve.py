"""The decoding model's operators against their definitions in 64 bits.

Tolerances are bounds on the roundings that the operators state:
  angle   the turn is rounded to float32 in half turns (2^-24 of at most pi),
          sincospi and two products and a sum add a few roundings: 5e-7 of |a| + |b|
  store   half a unit in the last place, relative: 2^-24 (float32, 24 significant
          bits), 2^-8 (bfloat16, 8) and 2^-4 (8-bit, 4; below 2^-6 2^-10 absolute)
  score   a dot product of D terms in float32: (D + 2) 2^-24 sum |q k| scale
  weight  exp of a score off by d is off by 2 d; rounded to bfloat16 2^-8, to
          float16 2^-11 (below 2^-14 2^-25 absolute); sums of n terms n 2^-24
"""
import math

import pytest
import torch

import paper_2608_13226_gb300 as cp

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
BF16, F32 = torch.bfloat16, torch.float32
ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, E4M3: 2.0 ** -4}
FLOOR = {F32: 0.0, BF16: 2.0 ** -134, E4M3: 2.0 ** -10}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_13226_gb300 import build
    build.build()
    cp.load()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def wide(x):
    return x.float().double() if x.dtype == E4M3 else x.double()


def turned(x, pos, f, layout, scale=1.0, back=False):
    """(result, |a| + |b| of each component's pair) in 64 bits; x [..., heads, D], pos [...]."""
    x, n = wide(x), f.numel()
    ang = pos.double()[..., None, None] * f
    c, s = ang.cos() * scale, ang.sin() * (-scale if back else scale)
    i, j = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b, y, mag = x[..., i], x[..., j], x.clone(), torch.zeros_like(x)
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    mag[..., i] = mag[..., j] = (a.abs() + b.abs()) * abs(scale)
    return y, mag


def assert_stored(got, want, extra, what):
    """got is want rounded to its type, want being known up to `extra`."""
    ulp, floor = ULP[got.dtype], FLOOR[got.dtype]
    err = (wide(got) - want).abs()
    tol = ulp * (want.abs() + extra) + extra + floor
    assert bool((err <= tol).all()), f"{what}: {(err - tol).max().item():.3g} over, err {err.max().item():.3g}"


def freq(n, base=1e4):
    return (base ** (-torch.arange(n, dtype=torch.float64) / max(n, 1))).cuda()


# ------------------------------------------------------------------ rotary
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,T,H,D,rot", [(1, 1, 1, 2, 2), (1, 3, 1, 128, 128), (2, 17, 7, 64, 64), (1, 33, 5, 80, 40), (3, 5, 2, 96, 20),
                                         (1, 4, 3, 256, 256), (1, 9, 2, 6, 4), (1, 2, 3, 7, 2), (2, 1, 28, 128, 64), (1, 2, 2, 16, 0),
                                         (1, 300, 40, 128, 128), (1, 1, 2, 2050, 2050), (1, 70001, 1, 8, 8)])
def test_rotary(B, T, H, D, rot, dtype, layout):
    g = gen(B * 1000 + T + D)
    x = randn(g, B, T, H, D, dtype=dtype)
    pos = torch.randint(0, 1 << 20, (B, T), generator=g, device="cuda")
    f = freq(rot // 2)
    for back in (False, True):
        y = cp.coverprune_rotary(x, pos, f, layout=layout, scale=1.25, inverse=back)
        want, mag = turned(x, pos, f, layout, 1.25, back)
        assert_stored(y, want, 5e-7 * mag, "rotary")
        assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,H,D,rot", [(100003, 1, 128, 128), (90001, 2, 64, 64), (50000, 1, 80, 80), (100000, 3, 48, 36),
                                       (20011, 1, 1100, 1100), (20000, 2, 256, 256)])
def test_rotary_many_tokens_of_few_heads(T, H, D, rot, dtype, layout):
    """Runs of tokens over many stages, whose angles outweigh their rows."""
    g = gen(T)
    x = randn(g, 1, T, H, D, dtype=dtype)
    pos = torch.randint(0, 1 << 20, (1, T), generator=g, device="cuda")
    y = cp.coverprune_rotary(x, pos, freq(rot // 2), layout=layout)
    want, mag = turned(x, pos, freq(rot // 2), layout)
    assert_stored(y, want, 5e-7 * mag, "rotary")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,shift", [(64, 0), (64, 1), (64, 4), (80, 2), (128, 8)])
def test_rotary_strides(D, shift, dtype):
    """Views of a fused projection at several alignments, heads before tokens,
    shared positions, two tensors in one launch, and in place."""
    g, f = gen(D + shift), freq(D // 2)
    T, Hq, Hk = 37, 6, 2
    flat = randn(g, 2 * T * (Hq + 2 * Hk) * (D + 8) + shift, dtype=dtype)[shift:].view(2, T, Hq + 2 * Hk, D + 8)
    q, k = flat[:, :, :Hq, :D], flat[:, :, Hq:Hq + Hk, :D]
    pos = torch.randint(-5000, 5000, (T,), generator=g, device="cuda")
    yq, yk = cp.coverprune_rotary([q, k], pos, f)
    for x, y in ((q, yq), (k, yk)):
        want, mag = turned(x, pos.expand(2, T), f, "half")
        assert_stored(y, want, 5e-7 * mag, "fused")
    hf = q.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    y = cp.coverprune_rotary(hf, pos, f)
    assert torch.equal(y, yq)
    assert torch.equal(cp.coverprune_rotary(q[1], pos, f), yq[1])
    rest = flat.clone()
    r = cp.coverprune_rotary([q, k], pos, f, out=[q, k])
    assert r[0] is q and torch.equal(q, yq) and torch.equal(k, yk)
    assert torch.equal(flat[:, :, Hq + Hk:], rest[:, :, Hq + Hk:]) and torch.equal(flat[..., D:], rest[..., D:])


def test_rotary_far_positions():
    """Positions up to 2^40 and negative ones: the angle is reduced exactly. In
    Python integers: turns = frac(f / 2 pi) in 80 bits."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    turn = 2 * Decimal("3.14159265358979323846264338327950288419716939937510")
    f = freq(32)
    pos = torch.tensor([0, 1, -1, 4097, (1 << 31) + 3, (1 << 40) + 12345, -(1 << 40)], device="cuda")
    x = torch.zeros(len(pos), 1, 64, device="cuda")
    x[..., :32] = 1.0  # half layout: the result is (cos, sin)
    y = cp.coverprune_rotary(x, pos, f).double().cpu()
    for i, p in enumerate(pos.tolist()):
        for j, fj in enumerate(f.tolist()):
            t = Decimal(p) * Decimal(fj) / turn
            a = float((t - t.to_integral_value()) * turn)
            # the speed in turns is a float64 product: off by up to 2^-53 of |t| turns, and 2^-64 |p|
            tol = 5e-7 + 2 * math.pi * (2 * abs(float(t)) * 2.0 ** -53 + abs(p) * 2.0 ** -64)
            assert abs(y[i, 0, j] - math.cos(a)) <= tol and abs(y[i, 0, j + 32] - math.sin(a)) <= tol


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient(layout):
    """Against the formula's transpose by differences: the rotation is linear, so
    <g, R(x + h d) - R(x)> / h = <R^T g, d> but for rounding."""
    g, T, H, D, rot = gen(5), 50, 3, 64, 48
    x, d, up = randn(g, T, H, D), randn(g, T, H, D), randn(g, T, H, D)
    pos, f = torch.arange(T, device="cuda") * 7, freq(rot // 2)
    R = lambda t, **kw: cp.coverprune_rotary(t, pos, f, layout=layout, scale=0.75, **kw).double()
    h = 2.0 ** -3
    num = (up.double() * (R(x + h * d) - R(x))).sum() / h
    got = (R(up, inverse=True) * d.double()).sum()
    n = T * H * D
    # each of n terms is off by 5e-7 (|a| + |b|) over h, signs as they fall: 5 sigma of n such errors
    assert abs(num - got) <= 5 * math.sqrt(n) * 4 * 5e-7 / h


def test_rotary_refuses_on_gpu():
    x, pos, f = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), freq(32)
    for bad in (dict(layout="other"), dict(out=torch.zeros(4, 2, 32, device="cuda")), dict(out=x.bfloat16())):
        with pytest.raises(ValueError):
            cp.coverprune_rotary(x, pos, f, **bad)
    for a in ((x, pos[:3], f), (x, pos, freq(33)), (x[0], pos, f), (x.transpose(1, 2), pos, f), ([], pos, f), ([x, x[:3]], pos, f)):
        with pytest.raises(ValueError):
            cp.coverprune_rotary(*a)
    for a in ((x, pos.int(), f), (x, pos, f.float()), (x.half(), pos, f)):
        with pytest.raises(TypeError):
            cp.coverprune_rotary(*a)


# ------------------------------------------------------------------ append
def pool(g, pages, page, H, D, dtype, heads_first=False, junk=None):
    shape = (pages, H, page, D) if heads_first else (pages, page, H, D)
    x = torch.full(shape, junk, device="cuda") if junk is not None else torch.randn(shape, generator=g, device="cuda")
    x = (x * 60 if dtype == E4M3 else x).to(dtype)
    return x.permute(0, 2, 1, 3) if heads_first else x


def bits(t):
    return t.view({4: torch.int32, 2: torch.int16, 1: torch.uint8}[t.element_size()])


def check_append(seed, new, past, page, Hq, Hk, D, rot, dtype, cdt, heads_first=False, use_pos=True, layout="half", scales=False,
                 padding=0, starts=True):
    g = gen(seed)
    B, T = len(new), sum(new) + padding
    W = max(1, -(-max(p + n for p, n in zip(past, new)) // page))
    pages = B * W + 2
    table = torch.randperm(pages, generator=g, device="cuda")[:B * W].reshape(B, W).int()
    fused = randn(g, T, Hq + 2 * Hk, D, dtype=dtype)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hk], fused[:, Hq + Hk:]
    kc, vc = pool(g, pages, page, Hk, D, cdt, heads_first), pool(g, pages, page, Hk, D, cdt, heads_first)
    k0, v0 = kc.clone(), vc.clone()
    ks, vs = (0.01 + torch.rand(2, Hk, generator=g, device="cuda")) if scales else (None, None)
    st = torch.tensor([0] + new).cumsum(0).int().cuda() if starts else None
    lens = torch.tensor(past).int().cuda()
    pos = torch.randint(0, 100000, (T,), generator=g, device="cuda") if use_pos else None
    f = freq(rot // 2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = cp.coverprune_cache_append(k, v, kc, vc, table, lens, starts=st, pos=pos, inv_freq=f, layout=layout, q=q if Hq else None,
                                   k_scale=ks, v_scale=vs, status=status)
    assert int(status) == 0
    assert r["lens"].tolist() == [p + n for p, n in zip(past, new)] and lens.tolist() == past
    n = T - padding
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(new, device="cuda"))
    slot = torch.cat([torch.arange(p, p + m) for p, m in zip(past, new)]).cuda()
    at = (table.long()[seq, slot // page], slot % page)
    where = slot if pos is None else pos[:n]
    want, mag = turned(k[:n], where, f, layout)
    one = torch.ones(Hk, 1, device="cuda", dtype=torch.float64)
    a, b = (one, one) if ks is None else (ks.double()[:, None], vs.double()[:, None])
    top = 448.0 if cdt == E4M3 else math.inf
    # dividing by the scale rounds once more
    assert_stored(bits(kc)[at].view(cdt), (want / a).clamp(-top, top), (5e-7 * mag + 2.0 ** -23 * want.abs()) / a, "keys")
    assert_stored(bits(vc)[at].view(cdt), (wide(v[:n]) / b).clamp(-top, top), 2.0 ** -23 * wide(v[:n]).abs() / b, "values")
    if Hq:
        want, mag = turned(q[:n], where, f, layout)
        assert_stored(r["q"][:n], want, 5e-7 * mag, "queries")
    for c, c0 in ((kc, k0), (vc, v0)):  # nothing else was written
        other = torch.ones(c.shape[:2], dtype=torch.bool, device="cuda")
        other[at] = False
        assert torch.equal(bits(c)[other], bits(c0)[other])


@pytest.mark.parametrize("dtype,cdt", [(BF16, BF16), (F32, F32), (BF16, E4M3), (F32, E4M3)])
@pytest.mark.parametrize("D,rot,layout,page,hf", [(64, 64, "half", 16, False), (128, 128, "interleaved", 7, True),
                                                  (80, 40, "half", 1, False), (256, 64, "interleaved", 100, True),
                                                  (96, 20, "half", 33, False), (16, 0, "half", 4, False)])
def test_append(dtype, cdt, D, rot, layout, page, hf):
    check_append(D + page, [5, 0, 1, 63, 0], [0, 9, 40, 3, 0], page, 6, 3, D, rot, dtype, cdt, hf, True, layout, cdt == E4M3)
    check_append(D + page + 1, [1] * 9, [0, 1, 2, 15, 16, 31, 32, 99, 100], page, 4, 2, D, rot, dtype, cdt, hf, False, layout,
                 True, starts=False)


@pytest.mark.parametrize("dtype,cdt", [(BF16, BF16), (F32, F32), (BF16, E4M3)])
@pytest.mark.parametrize("Hq,Hk,D,rot,page,hf", [(1, 1, 128, 128, 16, False), (8, 8, 64, 64, 16, True), (3, 1, 80, 80, 7, False),
                                                 (2, 2, 112, 48, 64, False), (5, 1, 128, 64, 100, True), (0, 2, 32, 32, 3, False)])
def test_append_many_tokens(Hq, Hk, D, rot, page, hf, dtype, cdt):
    check_append(D + Hq, [9000, 0, 12345, 7001, 1], [3, 0, 100, 0, 77], page, Hq, Hk, D, rot, dtype, cdt, hf, scales=cdt == E4M3)


@pytest.mark.parametrize("dtype,cdt", [(BF16, BF16), (F32, F32), (BF16, E4M3)])
@pytest.mark.parametrize("D,rot", [(80, 20), (80, 40), (96, 24), (96, 72), (128, 8), (16, 12)])
def test_append_interleaved_part(D, rot, dtype, cdt):
    """Turned parts of an odd number of vectors."""
    check_append(D + rot, [5, 0, 40, 1], [0, 3, 9, 70], 16, 5, 2, D, rot, dtype, cdt, layout="interleaved", scales=cdt == E4M3)
    x = randn(gen(rot), 2, 700, 3, D, dtype=dtype)
    pos = torch.randint(0, 1 << 20, (2, 700), generator=gen(D), device="cuda")
    y = cp.coverprune_rotary(x, pos, freq(rot // 2), layout="interleaved", inverse=True)
    want, mag = turned(x, pos, freq(rot // 2), "interleaved", back=True)
    assert_stored(y, want, 5e-7 * mag, "rotary")
    assert torch.equal(y[..., rot:], x[..., rot:])


def test_no_tokens_at_all():
    """Tensors without an element, whose address is null."""
    f, kc, vc = freq(32), torch.zeros(4, 16, 2, 64, device="cuda"), torch.zeros(4, 16, 2, 64, device="cuda")
    table = torch.arange(4, device="cuda").int().view(2, 2)
    none = torch.empty(0, 2, 64, device="cuda")
    lens = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    for pos in (None, torch.empty(0, dtype=torch.int64, device="cuda")):
        r = cp.coverprune_cache_append(none, none, kc, vc, table, lens, starts=torch.zeros(3, dtype=torch.int32, device="cuda"),
                                       pos=pos, inv_freq=f, q=torch.empty(0, 6, 64, device="cuda"))
        assert r["lens"].tolist() == [3, 0] and r["q"].shape == (0, 6, 64)
    r = cp.coverprune_cache_append(none, none, kc, vc, table[:0], lens[:0], inv_freq=f, q=torch.empty(0, 6, 64, device="cuda"))
    assert r["lens"].shape == (0,)
    assert not bool(kc.any()) and not bool(vc.any())
    for shape in ((1, 0, 2, 64), (0, 5, 2, 64), (2, 3, 0, 64)):
        x = torch.empty(shape, device="cuda")
        assert cp.coverprune_rotary(x, torch.zeros(shape[:2], dtype=torch.int64, device="cuda"), f).shape == shape
    r = cp.coverprune_decode_attention(torch.empty(0, 4, 64, device="cuda"), kc, vc, table[:0], lens[:0], lse=True)
    assert r["out"].shape == (0, 4, 64) and r["lse"].shape == (0, 4)


def test_append_many_and_padding():
    check_append(1, [0] * 700 + [3] + [0] * 300 + [2, 1], [1] * 1003, 4, 0, 1, 64, 64, BF16, BF16, padding=3)
    check_append(2, [1] * 1500, [7] * 1500, 16, 2, 1, 64, 64, BF16, E4M3, starts=False, scales=True)
    check_append(3, [5000], [11], 16, 28, 4, 128, 128, BF16, BF16)
    check_append(4, [2], [3], 16, 300, 100, 64, 32, BF16, BF16)


def test_append_specials_and_saturation():
    """8 bits: beyond the largest value and infinities saturate, NaN stays NaN."""
    v = torch.tensor([1e9, -1e9, math.inf, -math.inf, math.nan, 448.0, 465.0, 0.0009], device="cuda").repeat(2)[None, None]
    pages = torch.zeros(2, 1, 1, 16, device="cuda").to(E4M3)
    vals = torch.zeros_like(pages)
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    cp.coverprune_cache_append(v, v, pages, vals, table, lens)
    got = vals[0, 0, 0].float().tolist()
    assert got[:4] == [448.0, -448.0, 448.0, -448.0] and math.isnan(got[4]) and got[5:8] == [448.0, 448.0, 0.0]
    assert pages[0, 0, 0].float().tolist()[:4] == got[:4]


def test_append_out_of_room_and_bad_pages():
    g = gen(1)
    B, page, W, H, D = 5, 4, 2, 2, 64
    kc, vc = pool(g, 6, page, H, D, BF16), pool(g, 6, page, H, D, BF16)
    k0, v0 = kc.clone(), vc.clone()
    table = torch.tensor([[0, 1], [2, 6], [3, -1], [4, 5], [0, 1]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([8, 4, 5, 7, -2], dtype=torch.int32, device="cuda")  # full; bad pages; one slot left; no length
    k, v = randn(g, B, H, D, dtype=BF16), randn(g, B, H, D, dtype=BF16)
    q = randn(g, B, 4, D, dtype=BF16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = cp.coverprune_cache_append(k, v, kc, vc, table, lens, inv_freq=freq(32), q=q, status=status)
    assert int(status) == cp.CP_EINVAL
    assert r["lens"].tolist()[:4] == [8, 5, 6, 8]
    assert torch.equal(vc[5, 3], v[3]) and torch.equal(kc[:5], k0[:5]) and torch.equal(vc[:5], v0[:5])
    assert torch.equal(vc[5, :3], v0[5, :3]) and torch.equal(kc[5, :3], k0[5, :3])
    want, mag = turned(q, lens.long(), freq(32), "half")
    assert_stored(r["q"][:4], want[:4], 5e-7 * mag[:4], "queries")  # queries are turned all the same


# ------------------------------------------------------------------ attention
def attention(q, kc, vc, table, lens, ks, vs, window, keep, scale):
    """(out, lse, bound on out, bound on lse) in 64 bits, a sequence at a time."""
    B, Hq, D = q.shape
    H, page = kc.shape[2], kc.shape[1]
    G = Hq // H
    out, lse = torch.zeros(B, Hq, D, dtype=torch.float64, device="cuda"), torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    dout, dlse = torch.zeros_like(out), torch.zeros_like(lse)
    weight = {F32: 0.0, BF16: 2.0 ** -8, E4M3: 2.0 ** -11}[kc.dtype]
    for b, n in enumerate(lens.tolist()):
        n = min(max(n, 0), table.shape[1] * page)
        j = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        if keep is not None:
            j = j[keep[b][j]]
        pg = table[b].long()[j // page]
        j, pg = j[(pg >= 0) & (pg < kc.shape[0])], pg[(pg >= 0) & (pg < kc.shape[0])]
        if not len(j):
            continue
        for h in range(H):
            k = wide(bits(kc)[pg, j % page, h].view(kc.dtype)) * (1 if ks is None else float(ks[h]))
            v = wide(bits(vc)[pg, j % page, h].view(vc.dtype)) * (1 if vs is None else float(vs[h]))
            qq = wide(q[b, h * G:(h + 1) * G])
            s = qq @ k.T * scale
            ds = ((D + 4) * 2.0 ** -24 * (qq.abs() @ k.abs().T) * abs(scale)).amax(-1, keepdim=True)
            L = s.logsumexp(-1, keepdim=True)
            p = (s - L).exp()
            out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] = p @ v, L[:, 0]
            some = 2 * ds + 2 * s.abs().amax(-1, keepdim=True) * 2.0 ** -23 + (len(j) + 16) * 2.0 ** -24
            dout[b, h * G:(h + 1) * G] = (weight + some) * (p @ v.abs())
            if kc.dtype == E4M3:
                dout[b, h * G:(h + 1) * G] += len(j) * 2.0 ** -25 * v.abs().amax() * (s.amax(-1, keepdim=True) - L).exp()
            dlse[b, h * G:(h + 1) * G] = (some + 2.0 ** -22 * (1 + L.abs()))[:, 0]
    return out, lse, dout, dlse


def check_decode(seed, lens, page, Hq, H, D, cdt, window=0, keep=None, heads_first=False, scales=False, junk=None, width=None,
                 sharp=1.0, scale=None, q_view=False):
    g = gen(seed)
    B, dt = len(lens), F32 if cdt == F32 else BF16
    W = width or max(1, -(-max(max(lens), 1) // page))
    pages = B * W + 2
    table = torch.randperm(pages, generator=g, device="cuda")[:B * W].reshape(B, W).int()
    kc, vc = pool(g, pages, page, H, D, cdt, heads_first), pool(g, pages, page, H, D, cdt, heads_first)
    kp = None
    if keep is not None:
        kp = torch.rand(B, W * page + 3, generator=g, device="cuda") < keep
        kp = kp[:, :W * page]
    if junk is not None:  # whatever is not visible holds infinities or NaN
        j = torch.arange(W * page, device="cuda")[None]
        n = torch.tensor(lens, device="cuda")[:, None]
        vis = (j < n) & (j >= n - (window or 1 << 40))
        if kp is not None:
            vis = vis & kp
        mark = torch.ones(pages, page, dtype=torch.bool, device="cuda")
        seq = torch.arange(B, device="cuda")[:, None].expand_as(vis)
        mark[table.long()[seq, j.expand_as(vis) // page][vis], (j.expand_as(vis) % page)[vis]] = False
        bad = torch.full((), junk, device="cuda").to(cdt)
        bits(kc)[mark] = bits(bad[None])[0]
        bits(vc)[mark] = bits(bad[None])[0]
    ks, vs = (0.005 + 0.02 * torch.rand(2, H, generator=g, device="cuda")) if scales else (None, None)
    q = (randn(g, B, Hq + 2, D + 8) * sharp).to(dt)[:, 1:Hq + 1, 4:D + 4] if q_view else (randn(g, B, Hq, D) * sharp).to(dt)
    lt = torch.tensor(lens, dtype=torch.int32, device="cuda")
    tb = torch.where(torch.arange(W, device="cuda")[None] * page < lt[:, None], table, -1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(window=window, keep=kp, k_scale=ks, v_scale=vs, lse=True, scale=scale, status=status)
    r = cp.coverprune_decode_attention(q, kc, vc, tb, lt, **kw)
    want, L, dout, dlse = attention(q, kc, vc, tb, lt, ks, vs, window, kp, D ** -0.5 if scale is None else scale)
    assert int(status) == 0
    assert_stored(r["out"], want, dout, "out")
    got = r["lse"].double()
    assert torch.equal(got == -math.inf, L == -math.inf)
    fine = L > -math.inf
    assert bool(((got - L).abs()[fine] <= dlse[fine]).all()), f"lse off by {(got - L).abs()[fine].max()}"
    assert bool((r["out"][~fine] == 0).all())
    again = cp.coverprune_decode_attention(q, kc, vc, tb, lt, ws=r["ws"], **kw)
    assert torch.equal(bits(again["out"]), bits(r["out"])) and torch.equal(again["lse"], r["lse"])
    return r


TYPES = [(BF16, False), (F32, False), (E4M3, True)]


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("Hq,H,D", [(1, 1, 64), (28, 4, 128), (8, 8, 128), (16, 2, 80), (9, 1, 256), (24, 2, 96), (33, 3, 64),
                                    (40, 2, 128), (64, 1, 32), (4, 4, 16), (12, 3, 112), (34, 2, 256)])
def test_decode_heads(Hq, H, D, cdt, scales):
    check_decode(Hq * D, [0, 1, 15, 16, 17, 130, 1000], 16, Hq, H, D, cdt, scales=scales)


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("page", [1, 3, 16, 64, 100, 1024])
@pytest.mark.parametrize("hf", [False, True])
def test_decode_pages(page, hf, cdt, scales):
    check_decode(page, [63, 64, 65, 255, 256, 257, 2, 700], page, 14, 2, 128, cdt, heads_first=hf, scales=scales, junk=math.nan)


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 500, 5000])
def test_decode_window(window, cdt, scales):
    check_decode(window, [0, 1, 64, 65, 449, 2000], 16, 8, 2, 64, cdt, window=window, scales=scales, junk=math.nan)


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("keep,window", [(0.0, 0), (0.02, 0), (0.15, 0), (0.5, 300), (0.97, 0), (1.0, 0)])
def test_decode_keep(keep, window, cdt, scales):
    check_decode(7, [0, 1, 40, 300, 2000, 517], 16, 14, 2, 128, cdt, window=window, keep=keep, scales=scales, junk=math.nan)
    check_decode(8, [1500], 7, 4, 1, 64, cdt, window=window, keep=keep, scales=scales, junk=math.nan, heads_first=True)


@pytest.mark.parametrize("cdt,scales", TYPES)
def test_decode_lengths(cdt, scales):
    check_decode(1, [50000], 64, 4, 2, 64, cdt, scales=scales)                   # one long sequence over the whole GPU
    check_decode(2, [1] * 300 + [0] * 50 + [2] * 51, 16, 4, 2, 64, cdt, scales=scales)
    check_decode(3, [7000, 3, 0, 900] * 40, 32, 8, 1, 128, cdt, scales=scales)    # ragged
    check_decode(4, [5], 16, 4, 2, 64, cdt, scales=scales, width=2000)           # a table far wider than the keys
    check_decode(5, [0], 16, 4, 2, 64, cdt, scales=scales)
    check_decode(6, [300] * 70, 16, 7, 1, 128, cdt, scales=scales, q_view=True)


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("Hq,H,D,page", [(14, 2, 128, 16), (2, 2, 64, 7), (12, 1, 80, 100), (4, 1, 256, 1), (20, 1, 96, 64)])
def test_decode_many_short(Hq, H, D, page, cdt, scales):
    """More query tiles than blocks: whole, with marks, a window that makes long ones short."""
    lens = [0, 1, 2, 15, 16, 17, 31, 100, 7, 0] * 40
    check_decode(D, lens, page, Hq, H, D, cdt, scales=scales, junk=math.nan)
    check_decode(D + 1, [3 * n for n in lens], page, Hq, H, D, cdt, scales=scales, keep=0.4, junk=math.nan, heads_first=True)
    check_decode(D + 2, [7 * n for n in lens], page, Hq, H, D, cdt, scales=scales, window=33, junk=math.nan, q_view=True)


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("Hq,H,D,page,keep", [(14, 2, 128, 16, 0.1), (8, 8, 64, 1, 0.5), (6, 2, 256, 100, 0.02)])
def test_decode_many_marked(Hq, H, D, page, keep, cdt, scales):
    """Many sequences of some hundred keys of which few are marked, and some none."""
    lens = [0, 1, 200, 517, 64, 333, 1000, 90] * (50 if H == 2 else 13)
    check_decode(D, lens, page, Hq, H, D, cdt, scales=scales, keep=keep, junk=math.nan, heads_first=True)
    check_decode(D + 1, lens, page, Hq, H, D, cdt, scales=scales, keep=keep, window=400, junk=math.nan)


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("Hq,H,D,page", [(14, 2, 128, 16), (1, 1, 64, 7), (12, 1, 256, 100), (24, 2, 80, 1), (4, 4, 16, 64)])
def test_decode_few_long(Hq, H, D, page, cdt, scales):
    """Few query tiles, which clusters of blocks share, at lengths that leave some of them
    nothing: whole, with marks and a window."""
    for lens in ([257], [1000, 0, 3], [300, 2000, 1, 17, 999]):
        check_decode(D, lens, page, Hq, H, D, cdt, scales=scales, junk=math.nan)
        check_decode(D + 1, lens, page, Hq, H, D, cdt, scales=scales, keep=0.3, junk=math.nan, heads_first=True)
        check_decode(D + 2, lens, page, Hq, H, D, cdt, scales=scales, window=290, junk=math.nan, q_view=True)


@pytest.mark.parametrize("cdt,scales", TYPES)
@pytest.mark.parametrize("Hq,H,D", [(14, 2, 128), (3, 3, 64), (12, 1, 256), (40, 2, 80)])
@pytest.mark.parametrize("most", [1, 7, 8, 9, 16, 17, 32, 33, 64])
def test_decode_few_tiny(most, Hq, H, D, cdt, scales):
    """Few query tiles of hardly any keys, on both sides of a tile and of two."""
    lens = [most, 0, max(most - 1, 1), 1, most]
    check_decode(most, lens, 1, Hq, H, D, cdt, scales=scales, junk=math.nan)
    check_decode(most + 1, [3 * n for n in lens], 7, Hq, H, D, cdt, scales=scales, window=most, keep=0.6, junk=math.inf,
                 heads_first=True, q_view=True)


@pytest.mark.parametrize("cdt", [BF16, F32, E4M3])
def test_decode_empty_table(cdt):
    g = gen(3)
    kc, vc = pool(g, 4, 16, 2, 64, cdt), pool(g, 4, 16, 2, 64, cdt)
    q = randn(g, 3, 4, 64, dtype=F32 if cdt == F32 else BF16)
    table = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    r = cp.coverprune_decode_attention(q, kc, vc, table, torch.tensor([0, 5, 100], dtype=torch.int32, device="cuda"), lse=True)
    assert bool((r["out"] == 0).all()) and bool((r["lse"] == -math.inf).all())


@pytest.mark.parametrize("cdt,scales", TYPES)
def test_decode_sharp_and_scaled(cdt, scales):
    """Scores in the hundreds (one key takes all), all alike, and a negative scale."""
    check_decode(1, [400, 1], 16, 8, 2, 64, cdt, scales=scales, sharp=300.0)
    check_decode(2, [400, 1], 16, 8, 2, 64, cdt, scales=scales, sharp=1e-4)
    check_decode(3, [400, 1], 16, 8, 2, 64, cdt, scales=scales, scale=-0.5)
    check_decode(4, [400, 1], 16, 8, 2, 64, cdt, scales=scales, scale=0.0)
    check_decode(5, [333], 16, 8, 2, 64, cdt, scales=scales, sharp=1e-30)


@pytest.mark.parametrize("cdt,scales", TYPES)
def test_decode_visible_specials(cdt, scales):
    """NaN in a visible value reaches its component of the output, and no other
    sequence or component."""
    g, dt = gen(1), F32 if cdt == F32 else BF16
    kc, vc = pool(g, 8, 16, 2, 64, cdt), pool(g, 8, 16, 2, 64, cdt)
    table = torch.arange(8, device="cuda").int().view(2, 4)
    lens = torch.tensor([64, 50], dtype=torch.int32, device="cuda")
    bits(vc)[1, 3, 1, 5] = bits(torch.full((1,), math.nan, device="cuda").to(cdt))[0]
    q = randn(g, 2, 4, 64, dtype=dt)
    out = cp.coverprune_decode_attention(q, kc, vc, table, lens)["out"]
    want = torch.zeros(2, 4, 64, dtype=torch.bool, device="cuda")
    want[0, 2:, 5] = True
    assert torch.equal(out.isnan(), want)


def test_decode_bad_pages_and_lengths():
    g = gen(2)
    kc, vc = pool(g, 8, 16, 2, 64, BF16), pool(g, 8, 16, 2, 64, BF16)
    table = torch.tensor([[0, 8, 1], [2, -5, 3], [4, 5, 6], [2000000000, -2000000000, 9]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([40, 48, 1 << 30, 48], dtype=torch.int32, device="cuda")
    q = randn(g, 4, 4, 64, dtype=BF16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = cp.coverprune_decode_attention(q, kc, vc, table, lens, lse=True, status=status)
    assert int(status) == cp.CP_EINVAL
    want, L, dout, dlse = attention(q, kc, vc, table, lens, None, None, 0, None, 64 ** -0.5)
    assert_stored(r["out"], want, dout, "out")
    assert r["lse"][3].tolist() == [-math.inf] * 4
    status.zero_()
    lens[:] = torch.tensor([16, 16, -3, 0])
    r = cp.coverprune_decode_attention(q, kc, vc, table, lens, lse=True, status=status)
    assert int(status) == 0 and bool((r["out"][2:] == 0).all())


@pytest.mark.parametrize("cdt,scales", TYPES)
def test_offsets_past_32_bits(cdt, scales):
    """A cache whose rows lie beyond 2^32 bytes and 2^31 elements."""
    g, dt = gen(3), F32 if cdt == F32 else BF16
    page, H, D = 256, 8, 128
    pages = (1 << 31) // (page * H * D) + 40
    kc, vc = (torch.zeros(pages, page, H, D, dtype=torch.uint8 if cdt == E4M3 else cdt, device="cuda") for _ in "kv")
    kc, vc = kc.view(cdt), vc.view(cdt)
    top = torch.arange(pages - 8, pages, device="cuda").int().view(2, 4)
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    k, v = randn(g, 2 * 700, H, D, dtype=dt), randn(g, 2 * 700, H, D, dtype=dt)
    starts = torch.tensor([0, 700, 1400], dtype=torch.int32, device="cuda")
    one = torch.full((H,), 0.02, device="cuda") if scales else None
    lens = cp.coverprune_cache_append(k, v, kc, vc, top, lens, starts=starts, k_scale=one, v_scale=one)["lens"]
    assert lens.tolist() == [700, 700]
    assert_stored(bits(vc)[pages - 8, :256].view(cdt), wide(v[:256]) / (0.02 if scales else 1.0), wide(v[:256]).abs() * 1e-6 * 50, "v")
    q = randn(g, 2, 16, D, dtype=dt)
    r = cp.coverprune_decode_attention(q, kc, vc, top, lens, k_scale=one, v_scale=one)
    want, _, dout, _ = attention(q, kc, vc, top, lens, one, one, 0, None, D ** -0.5)
    assert_stored(r["out"], want, dout, "out")
    assert int(bits(kc)[:pages - 8].count_nonzero()) == 0


def test_decode_refuses_on_gpu():
    g = gen(4)
    kc, vc = pool(g, 4, 16, 2, 64, BF16), pool(g, 4, 16, 2, 64, BF16)
    table, lens = torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    q = randn(g, 3, 4, 64, dtype=BF16)
    ok = dict(q=q, k_cache=kc, v_cache=vc, table=table, lens=lens)
    cp.coverprune_decode_attention(**ok)
    keep = torch.ones(3, 16, dtype=torch.bool, device="cuda")
    cp.coverprune_decode_attention(**ok, keep=keep)
    for bad in (dict(v_cache=vc[:2]), dict(v_cache=vc.float()), dict(q=q[:2]), dict(q=q[..., :32]), dict(lens=lens[:2]),
                dict(keep=keep[:, :15]), dict(out=q[:2]), dict(table=table[:, 0]), dict(k_scale=torch.ones(3, device="cuda"))):
        with pytest.raises(ValueError):
            cp.coverprune_decode_attention(**{**ok, **bad})
    for bad in (dict(lens=lens.long()), dict(table=table.long()), dict(keep=keep.int()), dict(q=q.half())):
        with pytest.raises(TypeError):
            cp.coverprune_decode_attention(**{**ok, **bad})
    for bad, st in ((dict(q=randn(g, 3, 3, 64, dtype=BF16)), cp.CP_EINVAL), (dict(q=q.float()), cp.CP_EUNSUPPORTED),
                    (dict(window=-1), cp.CP_EINVAL), (dict(ws=torch.empty(8, dtype=torch.uint8, device="cuda")), cp.CP_EWORKSPACE)):
        with pytest.raises(cp.CoverPruneError) as e:
            cp.coverprune_decode_attention(**{**ok, **bad})
        assert e.value.status == st
    wide_pool = pool(g, 1, 16, 2, 64, BF16).expand(4, 16, 2, 64)
    with pytest.raises(ValueError):
        cp.coverprune_decode_attention(**ok, out=q[:1].expand(3, 4, 64))
    with pytest.raises(ValueError):
        cp.coverprune_cache_append(q[:, :2], q[:, :2], wide_pool, wide_pool, table, lens)
    cp.coverprune_decode_attention(**{**ok, "k_cache": wide_pool, "v_cache": wide_pool})  # only read
    k = randn(g, 3, 2, 64, dtype=BF16)
    for bad in (dict(v=k[:2]), dict(lens=lens[:2]), dict(k=k[:2], v=k[:2]), dict(q=q[:2]), dict(q=q.float()),
                dict(starts=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(new_lens=lens[:2])):
        with pytest.raises(ValueError):
            cp.coverprune_cache_append(**{**dict(k=k, v=k, k_cache=kc, v_cache=vc, table=table, lens=lens), **bad})
    with pytest.raises(cp.CoverPruneError):
        cp.coverprune_cache_append(k, k, kc, vc, table, lens, new_lens=lens)


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("cdt", [BF16, F32, E4M3])
def test_prompt_then_tokens_on_a_stream(cdt):
    """A ragged prompt and five tokens through the cache equal the attention over
    the keys and values as they were given, on a stream of the caller's and
    with one launch after another waiting for nothing else."""
    dt = F32 if cdt == F32 else BF16
    g = gen(9)
    B, Hq, H, D, page, W = 3, 8, 2, 64, 8, 20
    new = [100, 1, 37]
    f = freq(32)
    one = torch.full((H,), 0.02, device="cuda") if cdt == E4M3 else None
    kc, vc = pool(g, B * W, page, H, D, cdt, junk=math.nan), pool(g, B * W, page, H, D, cdt, junk=math.nan)
    table = torch.randperm(B * W, generator=g, device="cuda").int().view(B, W)
    k, v = randn(g, sum(new), H, D, dtype=dt), randn(g, sum(new), H, D, dtype=dt)
    starts = torch.tensor([0, 100, 101, 138], dtype=torch.int32, device="cuda")
    steps = [(randn(g, B, Hq, D, dtype=dt), randn(g, B, H, D, dtype=dt), randn(g, B, H, D, dtype=dt)) for _ in range(5)]
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), []
    with torch.cuda.stream(side):
        n, ws = cp.coverprune_cache_append(k, v, kc, vc, table, lens, starts=starts, inv_freq=f, k_scale=one, v_scale=one)["lens"], None
        for q, k1, v1 in steps:
            a = cp.coverprune_cache_append(k1, v1, kc, vc, table, n, inv_freq=f, q=q, k_scale=one, v_scale=one)
            n = a["lens"]
            r = cp.coverprune_decode_attention(a["q"], kc, vc, table, n, k_scale=one, v_scale=one, ws=ws)
            ws = r["ws"]
            got.append(r["out"])
    side.synchronize()
    assert n.tolist() == [105, 6, 42]
    for b in range(B):
        ks, vs, at = [k[starts[b]:starts[b + 1]]], [v[starts[b]:starts[b + 1]]], 0
        for i, (q, k1, v1) in enumerate(steps):
            ks.append(k1[b:b + 1])
            vs.append(v1[b:b + 1])
            kk, vv = torch.cat(ks), wide(torch.cat(vs))
            m = len(kk)
            kk = turned(kk, torch.arange(m, device="cuda"), f, "half")[0]
            qq = turned(q[b:b + 1], torch.tensor([m - 1], device="cuda"), f, "half")[0][0]
            s = torch.einsum("hgd,jhd->hgj", qq.view(H, Hq // H, D), kk) * D ** -0.5
            want = torch.einsum("hgj,jhd->hgd", s.softmax(-1), vv).reshape(Hq, D)
            # queries and keys are rounded (u a component): scores are off by 2 u sum |q k| scale at most,
            # weights by twice that, values and outputs by u
            u = ULP[cdt if cdt == E4M3 else dt]
            mag = (qq.abs().view(H, Hq // H, D).unsqueeze(2) * kk.abs().permute(1, 0, 2).unsqueeze(1)).sum(-1).amax() * D ** -0.5
            tol = (4 * u * mag + 3 * u + 1e-5) * vv.abs().amax()
            assert bool(((got[i][b].double() - want).abs() <= tol).all())


def test_graph_capture():
    """A decode step (append with the query's rotation, attention) in a CUDA graph,
    replayed with other lengths: nothing depends on the host."""
    g = gen(11)
    B, Hq, H, D, page, W = 4, 8, 2, 128, 16, 40
    kc, vc = pool(g, B * W, page, H, D, BF16), pool(g, B * W, page, H, D, BF16)
    table, f = torch.arange(B * W, device="cuda").int().view(B, W), freq(64)
    q, k, v = randn(g, B, Hq, D, dtype=BF16), randn(g, B, H, D, dtype=BF16), randn(g, B, H, D, dtype=BF16)
    lens = torch.tensor([3, 0, 600, 100], dtype=torch.int32, device="cuda")
    new, qo, out = torch.empty_like(lens), torch.empty_like(q), torch.empty_like(q)

    def step(ws=None):
        cp.coverprune_cache_append(k, v, kc, vc, table, lens, inv_freq=f, q=q, new_lens=new, q_out=qo)
        return cp.coverprune_decode_attention(qo, kc, vc, table, new, out=out, ws=ws)["ws"]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ws = step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ws)
    for n in ([1, 2, 3, 4], [639, 200, 0, 16]):
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        q.copy_(randn(g, B, Hq, D, dtype=BF16))
        graph.replay()
        want, _, dout, _ = attention(qo, kc, vc, table, new, None, None, 0, None, D ** -0.5)
        assert_stored(out, want, dout, "graph")
        assert new.tolist() == [x + 1 for x in n]
