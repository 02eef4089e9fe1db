"""The decoding model's operators at the edges of what they take: arguments that
are refused, values at the ends of a type, and the bounds that the header states."""
import math

import pytest
import torch

import paper_2608_13226_gb300 as cp
from test_gpu_serve import ULP, assert_stored, attention, freq, gen, pool, randn, turned

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
BF16, F32 = torch.bfloat16, torch.float32
# lengths that are dealt out in each way: a warp a query tile (few keys; many
# sequences), a block each, a cluster each, one line
LENGTHS = {"tiny": [5, 9, 1], "warps": [300, 41] * 200, "blocks": [200, 130, 256], "clusters": [1500, 3], "line": [700] * 200}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_13226_gb300 import build
    build.build()
    cp.load()


def test_workspace_that_is_not_dense_is_refused():
    """Views that claim more bytes than they hold, or whose bytes lie apart: the call
    writes a run of bytes from the first on."""
    kc, vc = torch.zeros(2, 4, 16, 2, 64, dtype=BF16, device="cuda")
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 4, 64, dtype=BF16, device="cuda")
    ws = cp.coverprune_decode_attention(q, kc, vc, table, lens)["ws"]
    n = ws.numel()
    room = torch.zeros(2 * n, dtype=torch.uint8, device="cuda")
    for bad in (room[:1].expand(n), room[::2], room.view(2, n).t()):
        with pytest.raises(ValueError):
            cp.coverprune_decode_attention(q, kc, vc, table, lens, ws=bad)
    assert not bool(room.any())
    cp.coverprune_decode_attention(q, kc, vc, table, lens, ws=room.view(2, n)[0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", LENGTHS.values(), ids=list(LENGTHS))
def test_infinite_values(lens, dtype):
    """An infinite visible value makes its component infinite, two of both signs NaN, and no
    other component notices."""
    g, B, H, G, D, page = gen(len(lens)), len(lens), 2, 3, 64, 16
    W = -(-max(lens) // page)
    kc, vc = pool(g, B * W, page, H, D, dtype), pool(g, B * W, page, H, D, dtype)
    table = torch.randperm(B * W, generator=g, device="cuda").int().view(B, W)
    n = torch.tensor(lens, device="cuda")
    # a key of each sequence, another one, and what they hold in components 5, 9 and 40
    one = (torch.rand(B, generator=g, device="cuda") * n).long()
    other = (one + 1 + (torch.rand(B, generator=g, device="cuda") * (n - 1)).long()) % n
    seq = torch.arange(B, device="cuda")
    for key, at, x in ((one, 5, math.inf), (other, 9, -math.inf), (one, 40, math.inf), (other, 40, -math.inf)):
        some = n > 1 if at == 40 else n > 0
        vc[table.long()[seq, key // page][some], (key % page)[some], 1, at] = x
    q, lens = randn(g, B, G * H, D, dtype=dtype), n.int()
    got = cp.coverprune_decode_attention(q, kc, vc, table, lens)["out"].double()
    want, _, dout, _ = attention(q, kc, vc, table, lens, None, None, 0, None, D ** -0.5)
    assert bool((want[:, G:, 5] == math.inf).all()) and bool((want[:, G:, 9] == -math.inf).all())
    assert bool(want[n > 1][:, G:, 40].isnan().all()) and bool(want[:, :G].isfinite().all())
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.isinf() * got.sign(), want.isinf() * want.sign())
    fine = want.isfinite()
    assert bool(((got - want).abs() <= ULP[dtype] * (want.abs() + dout) + dout)[fine].all())


@pytest.mark.parametrize("apart", [4.0, 11.0, 15.0, 17.35, 20.0])
@pytest.mark.parametrize("cdt,n", [(E4M3, 30), (E4M3, 250), (E4M3, 5000), (E4M3, 200001), (BF16, 200001), (F32, 200001)])
def test_many_weak_keys_beside_a_strong_one(cdt, n, apart):
    """What n equal keys weigh together beside one that is `apart` (natural units) above each."""
    D, page, dt = 64, 64, F32 if cdt == F32 else BF16
    W = -(-n // page)
    kc, vc = torch.zeros(2, W, page, 1, D, device="cuda")
    strong = n // 3
    kc[strong // page, strong % page, 0, 0] = 1.0     # a score of 1 times the scale, where the others have 0
    vc[..., 0], vc[..., 1] = 1.0, 1.0
    vc[strong // page, strong % page, 0, 1] = 0.0     # component 0 is 1 whatever the weights, 1 is the weak keys' share
    q = torch.zeros(1, 1, D, dtype=dt, device="cuda")
    q[..., 0] = 1.0
    table = torch.arange(W, device="cuda").int()[None]
    r = cp.coverprune_decode_attention(q, kc.to(cdt), vc.to(cdt), table, torch.tensor([n], dtype=torch.int32, device="cuda"),
                                       scale=apart, lse=True)
    each = math.exp(-apart)
    total = 1 + (n - 1) * each
    share = (n - 1) * each / total
    # a weight is off by 2^-11 of itself and 2^-(25 + 7) of the largest (8 bits), 2^-16 (bfloat16); scores below 32 in float32,
    # in units of log 2, give 2^-18 at most, sums of n terms n 2^-24 at most (but for very few warps they are far shorter)
    part = {E4M3: 2.0 ** -11, BF16: 2.0 ** -16, F32: 0.0}[cdt] + 2.0 ** -17 + min(n, 4096) * 2.0 ** -24
    floor = 2.0 ** -32 * n / total if cdt == E4M3 else 0.0
    got, want = r["out"][0, 0].double().tolist(), [1.0, share]
    for i in range(2):
        off = part * want[i] + floor
        assert abs(got[i] - want[i]) <= off + ULP[dt] * (want[i] + off), (i, got[i], want[i])
    assert abs(float(r["lse"]) - (apart + math.log(total))) <= part + 2.0 ** -22 * 32


@pytest.mark.parametrize("cdt", [BF16, F32, E4M3])
@pytest.mark.parametrize("lens", LENGTHS.values(), ids=list(LENGTHS))
def test_scores_near_the_lowest_number(lens, cdt):
    """Keys that all score about -1.3e38, or -2.2e38: they are visible, alike ones weigh the
    same, and one that is above the others takes all."""
    g, dt, B, H, G, D, page = gen(len(lens)), F32 if cdt == F32 else BF16, len(lens), 2, 3, 64, 16
    W = -(-max(lens) // page)
    vc = pool(g, B * W, page, H, D, cdt)
    k = torch.zeros(B * W, page, H, D, device="cuda")
    q = torch.zeros(B, G * H, D, device="cuda", dtype=dt)
    unit = 2.0 ** 63
    q[..., 0] = unit
    k[..., 0] = -16.0  # kv head 0: all alike; 1: the first key above the rest
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    table = torch.arange(B * W, device="cuda").int().view(B, W)
    k[:, :, 1, 0] = -28.0
    k[table[:, 0].long(), 0, 1, 0] = -16.0
    factor = 2.0 ** 60 if cdt != E4M3 else 1.0  # 8 bits take it as their scale
    ks = torch.full((H,), 2.0 ** 60, device="cuda") if cdt == E4M3 else None
    vs = torch.full((H,), 0.02, device="cuda") if cdt == E4M3 else None
    r = cp.coverprune_decode_attention(q, (k * factor).to(cdt), vc, table, n, scale=0.75, k_scale=ks, v_scale=vs, lse=True)
    score = -16.0 * 2.0 ** 123 * 0.75
    assert -1.4e38 < score < -1.2e38 and -28.0 * 2.0 ** 123 * 0.75 / math.log(2) > -3.4028e38
    v = vc.float().double() * (0.02 if cdt == E4M3 else 1.0)
    # weights of exactly 1, sums of n terms in float32, one product and quotient, 1 / 0.02 of 8 bits rounded once
    for b in range(0, B, max(1, B // 7)):
        m = lens[b]
        rows = v[table[b].long()].reshape(-1, H, D)[:m]
        for h, want, mag in ((0, rows[:, 0].mean(0), rows[:, 0].abs().mean(0)), (1, rows[0, 1], rows[0, 1].abs())):
            got, extra = r["out"][b, h * G:(h + 1) * G].double(), (m + 8) * 2.0 ** -24 * mag
            assert bool(((got - want).abs() <= ULP[dt] * (want.abs() + extra) + extra).all()), (b, h)
    assert bool(((r["lse"].double() - score).abs() <= 2.0 ** -22 * abs(score)).all())


@pytest.mark.parametrize("lens", LENGTHS.values(), ids=list(LENGTHS))
def test_bf16_weights_have_two_terms(lens):
    """Few keys that count and values of one sign, so that errors of weights do not average
    out: the output is one of the bfloat16 between the exact one less and plus 2^-16 of it.
    The same computed with weights of a single term is not, so the bound would notice it."""
    g, B, D, page = gen(len(lens)), len(lens), 64, 16
    W = -(-max(lens) // page)
    table = torch.arange(B * W, device="cuda").int().view(B, W)
    k = torch.zeros(B * W, page, 1, D, dtype=BF16, device="cuda")
    k[..., 0] = -300.0
    v = (1 + torch.rand(B * W, page, 1, D, generator=g, device="cuda")).bfloat16()
    q = torch.zeros(B, 1, D, dtype=BF16, device="cuda")
    q[..., 0] = 1.0
    want, single = torch.zeros(B, D, dtype=torch.float64, device="cuda"), torch.zeros(B, D, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        at = torch.randperm(n, generator=g, device="cuda")[:5]
        page_of = table[b].long()[at // page]
        score = (-3 * torch.rand(len(at), generator=g, device="cuda")).bfloat16()
        k[page_of, at % page, 0, 0] = score
        w = (score.double() - score.double().max()).exp()
        x = v[page_of, at % page, 0].double()
        want[b], single[b] = w @ x / w.sum(), w.bfloat16().double() @ x / w.sum()
    # a score is one product, scaled in float32 (below 8: 2^-21), exp2 within 2^-22, a few sums and a quotient; the rest weigh e^-297
    off = 2.0 ** -16 + 2.0 ** -19
    low, high = (want * (1 - off)).bfloat16(), (want * (1 + off)).bfloat16()
    got = cp.coverprune_decode_attention(q, k, v, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), scale=1.0)["out"][:, 0]
    assert bool(((low <= got) & (got <= high)).all())
    other = single.bfloat16()
    assert bool(((other < low) | (other > high)).any())


def test_rotary_angles_at_far_positions():
    """The angle is off by 2^-64 turns for each position and no more, at positive and negative
    speeds and positions, against decimals of 60 digits; 5e-7 for sine, cosine and a product."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    turn = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    g = torch.Generator().manual_seed(1)
    speeds = [1.0, -1.0, 3.7, -250.125, 1e-3, -1e-3, 1e-7, -1e-9] + (10 ** (-5 * torch.rand(24, generator=g, dtype=torch.float64))).tolist()
    f = torch.tensor(speeds, dtype=torch.float64, device="cuda")
    places = [1, -1, 8191, (1 << 31) + 3, -(1 << 31), (1 << 40) + 12345, -(1 << 40) - 7, (1 << 40) - 1]
    x = torch.zeros(len(places), 1, 64, device="cuda")
    x[..., :32] = 1.0  # half layout: the result is (cos, sin)
    y = cp.coverprune_rotary(x, torch.tensor(places, device="cuda"), f).double().cpu()
    for i, p in enumerate(places):
        off = 5e-7 + 2 * math.pi * abs(p) * 2.0 ** -64
        for j, s in enumerate(speeds):
            t = Decimal(p) * Decimal(s) / turn
            a = float((t - t.to_integral_value()) * turn)
            assert abs(y[i, 0, j] - math.cos(a)) <= off and abs(y[i, 0, j + 32] - math.sin(a)) <= off, (p, s)


@pytest.mark.parametrize("cdt", [BF16, F32, E4M3])
def test_rows_before_the_first_sequence_are_padding(cdt):
    """A part of a longer batch: its starts begin above 0, and what lies before is left alone."""
    g, dt, page, H, D = gen(5), F32 if cdt == F32 else BF16, 4, 2, 64
    kc, vc = pool(g, 9, page, H, D, cdt), pool(g, 9, page, H, D, cdt)
    k0, v0 = kc.clone(), vc.clone()
    table = torch.randperm(9, generator=g, device="cuda").int().view(3, 3)
    k, v, q = (randn(g, 15, h, D, dtype=dt) for h in (H, H, 6))
    lens = torch.tensor([5, 0, 2], dtype=torch.int32, device="cuda")
    starts = torch.tensor([3, 8, 8, 12], dtype=torch.int32, device="cuda")
    status, q_out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full_like(q, 7.0)
    r = cp.coverprune_cache_append(k, v, kc, vc, table, lens, starts=starts, q=q, q_out=q_out, status=status)
    assert r["lens"].tolist() == [10, 0, 6] and int(status) == 0
    rows = {(0, 5 + i): 3 + i for i in range(5)} | {(2, 2 + i): 8 + i for i in range(4)}
    for (b, j), t in rows.items():
        at = (int(table[b, j // page]), j % page)
        for c, c0, x in ((kc, k0, k), (vc, v0, v)):
            assert torch.equal(c[at].view(torch.uint8), x[t].to(cdt).view(torch.uint8))
            c0.view(torch.uint8)[at] = c[at].view(torch.uint8)
    for c, c0 in ((kc, k0), (vc, v0)):
        assert torch.equal(c.view(torch.uint8), c0.view(torch.uint8))
    assert torch.equal(q_out[3:12], q[3:12]) and bool((q_out[:3] == 7).all()) and bool((q_out[12:] == 7).all())


def test_a_negative_length_stays_negative():
    """Its tokens are skipped, so the sequence must not come to hold keys that were never written."""
    g, page, H, D = gen(6), 4, 2, 64
    kc, vc = pool(g, 6, page, H, D, BF16), pool(g, 6, page, H, D, BF16)
    k0 = kc.clone()
    table = torch.arange(6, device="cuda").int().view(3, 2)
    k = randn(g, 12, H, D, dtype=BF16)
    lens = torch.tensor([-2, 1, -1], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 6, 7, 12], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = cp.coverprune_cache_append(k, k, kc, vc, table, lens, starts=starts, status=status)
    assert int(status) == cp.CP_EINVAL and r["lens"].tolist() == [-2, 2, -1]
    assert torch.equal(kc[2, 1], k[6]) and torch.equal(kc[[0, 1, 4, 5]], k0[[0, 1, 4, 5]])
    out = cp.coverprune_decode_attention(randn(g, 3, 4, D, dtype=BF16), kc, vc, table, r["lens"])["out"]
    assert bool((out[[0, 2]] == 0).all()) and bool((out[1] != 0).any())


def test_status_without_an_element_is_refused():
    """Errors would go nowhere, though the caller asked for them."""
    kc, vc = torch.zeros(2, 4, 16, 2, 64, dtype=BF16, device="cuda")
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    q, none = torch.zeros(1, 2, 64, dtype=BF16, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        cp.coverprune_decode_attention(q, kc, vc, table, lens, status=none)
    with pytest.raises(ValueError):
        cp.coverprune_cache_append(q, q, kc, vc, table, lens, status=none)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary_is_part_of_autograd(dtype, layout, inverse):
    """The gradient through a call against autograd of the formula in 64 bits; of two tensors
    of which one wants it; of an expanded gradient; and the gradient's own."""
    g, f = gen(8), freq(24)
    x, other = randn(g, 2, 33, 5, 64, dtype=dtype).requires_grad_(), randn(g, 2, 33, 2, 64, dtype=dtype)
    pos = torch.randint(0, 1 << 20, (2, 33), generator=g, device="cuda")
    up = randn(g, 2, 33, 5, 64, dtype=dtype).requires_grad_()
    kw = dict(layout=layout, scale=1.25, inverse=inverse)
    y, z = cp.coverprune_rotary([x, other], pos, f, **kw)
    assert y.requires_grad and not z.requires_grad
    with torch.no_grad():
        assert torch.equal(y, cp.coverprune_rotary(x, pos, f, **kw)) and torch.equal(z, cp.coverprune_rotary(other, pos, f, **kw))
    got, = torch.autograd.grad(y, x, up, create_graph=True)
    wide = x.detach().double().requires_grad_()
    want, = torch.autograd.grad(turned(wide, pos, f, layout, 1.25, inverse)[0], wide, up.detach().double())
    mag = turned(up.detach(), pos, f, layout, 1.25)[1]
    assert got.dtype == dtype
    assert_stored(got.detach(), want, 5e-7 * mag, "gradient")
    # the gradient is linear in `up`, by the turn that the call itself makes
    w = randn(g, 2, 33, 5, 64, dtype=dtype)
    assert torch.equal(torch.autograd.grad(got, up, w)[0], cp.coverprune_rotary(w, pos, f, **kw))
    cp.coverprune_rotary(x, pos, f, **kw).sum().backward()
    assert torch.equal(x.grad, cp.coverprune_rotary(torch.ones_like(w), pos, f, layout=layout, scale=1.25, inverse=not inverse))
    with torch.no_grad():
        assert not cp.coverprune_rotary(x, pos, f, **kw).requires_grad


def test_rotary_gradient_by_differences():
    """Through autograd, of a function that is not linear: (R x)^2 / 2 summed with weights."""
    g, f, pos = gen(9), freq(32), torch.arange(40, device="cuda") * 5
    x, d, w = (randn(g, 40, 3, 64) for _ in range(3))
    value = lambda t: (w.double() * cp.coverprune_rotary(t, pos, f, scale=0.75).double() ** 2).sum() / 2
    x.requires_grad_()
    grad, = torch.autograd.grad(value(x), x)
    h = 2.0 ** -6
    with torch.no_grad():
        num = (value(x + h * d) - value(x - h * d)) / (2 * h)
        got = (grad.double() * d.double()).sum()
    # the function is quadratic: only roundings differ, 2^-22 of each of n terms of up to 5^3, signs as they fall, over h
    assert abs(num - got) <= 5 * math.sqrt(x.numel()) * 125 * 2.0 ** -22 / h


def test_what_gives_no_gradient_refuses_to_drop_one():
    g, D, H = gen(10), 64, 2
    kc, vc = pool(g, 4, 16, H, D, F32), pool(g, 4, 16, H, D, F32)
    table, lens = torch.arange(4, device="cuda").int().view(2, 2), torch.tensor([3, 5], dtype=torch.int32, device="cuda")
    k, q, f, pos = randn(g, 2, H, D), randn(g, 2, 4, D), freq(32), torch.tensor([3, 5], device="cuda")
    append = dict(k=k, v=k, k_cache=kc, v_cache=vc, table=table, lens=lens, inv_freq=f, q=q)
    attend = dict(q=q, k_cache=kc, v_cache=vc, table=table, lens=lens)
    keep = kc.clone()
    for call, args, names in ((cp.coverprune_cache_append, append, ("k", "v", "q", "k_cache", "inv_freq")),
                              (cp.coverprune_decode_attention, attend, ("q", "k_cache", "v_cache"))):
        for name in names:
            bad = {**args, name: args[name].detach().requires_grad_()}
            with pytest.raises(ValueError, match="gradient"):
                call(**bad)
            if name != "k_cache":
                with torch.no_grad():
                    call(**bad)
                    kc.copy_(keep)
    wanting = q.detach().clone().requires_grad_()
    for kw in (dict(x=wanting, out=torch.empty_like(q)), dict(x=q, out=wanting), dict(x=wanting, out=wanting)):
        with pytest.raises(ValueError, match="gradient"):
            cp.coverprune_rotary(kw.pop("x"), pos, f, **kw)
    with pytest.raises(ValueError, match="gradient"):
        cp.coverprune_rotary(q, pos, f.clone().requires_grad_())


def test_autograd_notices_what_is_written():
    """A tensor that autograd saved and a call then overwrote must not enter a gradient."""
    g, D, H = gen(11), 64, 2
    kc, vc = pool(g, 4, 16, H, D, F32), pool(g, 4, 16, H, D, F32)
    table, lens = torch.arange(4, device="cuda").int().view(2, 2), torch.tensor([3, 5], dtype=torch.int32, device="cuda")
    k, q, f, pos = randn(g, 2, H, D), randn(g, 2, 4, D), freq(32), torch.tensor([3, 5], device="cuda")
    q_out, out = torch.zeros_like(q), torch.zeros_like(q)
    new_lens, status = torch.zeros_like(lens), torch.zeros(1, dtype=torch.int32, device="cuda")
    one = torch.ones((), device="cuda", requires_grad=True)
    append = lambda: cp.coverprune_cache_append(k, k, kc, vc, table, lens, inv_freq=f, q=q, q_out=q_out, new_lens=new_lens, status=status)
    attend = lambda: cp.coverprune_decode_attention(q, kc, vc, table, lens, out=out, status=status)
    turn = lambda: cp.coverprune_rotary(q, pos, f, out=q)
    turns = lambda: cp.coverprune_rotary([q, k], pos, f, out=[q, k])
    for call, written, read in ((append, (kc, vc, q_out, new_lens, status), (k, q, lens, table)), (attend, (out, status), (q, kc, vc)),
                                (turn, (q,), (k,)), (turns, (q, k), (out,))):
        before = {id(t): t._version for t in (*written, *read)}
        call()
        assert all(t._version > before[id(t)] for t in written) and all(t._version == before[id(t)] for t in read)
        for t in (t for t in written if t.is_floating_point()):
            product = (one * t).sum()
            call()
            with pytest.raises(RuntimeError, match="inplace"):
                product.backward()
    with torch.inference_mode():
        kc, vc, out = kc.clone(), vc.clone(), out.clone()
        append(), attend()
    append(), attend()  # tensors made in inference mode have no versions


def test_lse_that_is_neither_true_nor_false():
    """What its truth raises comes through."""
    class Unclear:
        def __bool__(self):
            raise KeyError("unclear")

    kc, vc = torch.zeros(2, 4, 16, 2, 64, dtype=BF16, device="cuda")
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    with pytest.raises(KeyError):
        cp.coverprune_decode_attention(torch.zeros(1, 2, 64, dtype=BF16, device="cuda"), kc, vc, table, lens, lse=Unclear())
