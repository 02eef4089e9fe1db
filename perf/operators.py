"""The calls that a program makes once the visual tokens of a scene have been pruned and a language model decodes on the
kept ones: rotary positions at the kept tokens' own indices, the append of keys and values to a paged cache, and the
attention of one new token a sequence over that cache.

A case names one operator ("op"), its sizes and the options that the program would set.  `own` picks what `run` does: the
framework's entry points, or the same operators in elementary torch operations.  Heads are those of the feature widths
of the pruned scenes (3584 = 28 x 128, 1280 = 20 x 64 or 16 x 80, 256 = 4 x 64), lengths those of pruned and unpruned scenes
(1229 and 8192 tokens) with some text, and longer caches.
"""
import math

import torch

own = False

ROTARY, APPEND, ATTEND = "rotary", "append", "attend"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}
LARGEST = 448.0  # the largest e4m3 value


def _rotary(B, T, Hq, Hk, D, **options):
    c = {"op": ROTARY, "B": B, "T": T, "Hq": Hq, "Hk": Hk, "D": D, "rot": D, "layout": "half", "dtype": "bf16",
         "gradient": False, "heads_first": False, "span": 8192, "stretch": 1.0}
    c.update(options)
    return c


def _append(B, lo, hi, Hq, Hk, D, **options):
    c = {"op": APPEND, "B": B, "lo": lo, "hi": hi, "past": 0, "Hq": Hq, "Hk": Hk, "D": D, "rot": D, "layout": "half",
         "dtype": "bf16", "cache": "bf16", "page": 16, "heads_first": False, "span": 8192, "stretch": 1.0}
    c.update(options)
    return c


def _attend(B, lo, hi, Hq, Hk, D, **options):
    c = {"op": ATTEND, "B": B, "lo": lo, "hi": hi, "Hq": Hq, "Hk": Hk, "D": D, "dtype": "bf16", "cache": "bf16", "page": 16,
         "heads_first": False, "window": 0, "keep": 1.0}
    c.update(options)
    return c


def listed():
    return [
        # the prompt of the throughput batch: queries and keys of 32 scenes' kept tokens, rotated at their indices in the scene
        dict(_rotary(32, 1229, 28, 4, 128), name="rotary prompt"),
        # a training step's gradient through the rotation, heads before tokens, part of each head, neighbouring components paired
        dict(_rotary(2, 4096, 16, 16, 80, rot=40, layout="interleaved", dtype="f32", gradient=True, heads_first=True, span=4096),
             name="rotary gradient f32"),
        # one token of each of 32 sequences far into a context stretched by 8: latency
        dict(_rotary(32, 1, 28, 4, 128, span=1 << 20, stretch=8.0), name="rotary token"),
        # the same prompt on its way into the cache: ragged kept sets, keys rotated, values as they are, queries rotated as well
        dict(_append(32, 900, 1500, 28, 4, 128), name="append prompt"),
        # one token of each of 64 sequences into an 8-bit cache: what every decoded token pays in every layer
        dict(_append(64, 1, 1, 28, 4, 128, cache="e4m3", past=1229, span=0, heads_first=True, page=32), name="append token e4m3"),
        # one scene alone after pruning, some text in: the latency between two words
        dict(_attend(1, 1500, 1500, 28, 4, 128), name="attend one scene"),
        # the throughput batch after pruning to 15%
        dict(_attend(32, 1229, 1741, 28, 4, 128), name="attend batch kept"),
        # the same batch unpruned, to show what pruning saves
        dict(_attend(32, 8192, 8704, 28, 4, 128), name="attend batch unpruned"),
        # one very long cache: nothing but the split over its length fills the GPU
        dict(_attend(1, 200001, 200001, 32, 8, 128, page=64), name="attend long"),
        # many sequences of very different lengths over an 8-bit cache, heads before slots in a page
        dict(_attend(128, 500, 16000, 16, 2, 128, cache="e4m3", page=32, heads_first=True), name="attend ragged e4m3"),
        # scenes pruned in place after their prefill: 15% of the cached rows are read, the others stay where they are
        dict(_attend(16, 8192, 8704, 28, 4, 128, keep=0.15), name="attend kept in place"),
        # a small model in 32 bits: empty and short sequences, pages of 7, a window
        dict(_attend(9, 0, 1100, 4, 4, 64, dtype="f32", cache="f32", page=7, window=500), name="attend f32 window"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice([ROTARY, APPEND, ATTEND, ATTEND])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    D = rng.choice([64, 80, 96, 128, 128, 256])
    Hk = rng.choice([1, 2, 3, 4, 8])
    Hq = Hk * rng.choice([1, 2, 4, 5, 7, 8, 12, 16])
    rot = rng.choice([D, D, D // 2, D // 4])
    rest = {"rot": rot, "layout": rng.choice(["half", "interleaved"]), "heads_first": rng.random() < 0.3,
            "stretch": rng.choice([1.0, 1.0, 4.0])}
    if op == ROTARY:
        B = _log(rng, 1, 64)
        T = _log(rng, 1, max(1, min(20000, 350000000 // (B * (Hq + Hk) * D * SIZE[dtype]))))
        return _rotary(B, T, Hq, Hk, D, dtype=dtype, gradient=rng.random() < 0.4, span=max(T, _log(rng, 100, 1 << 20)), **rest)
    page = rng.choice([1, 7, 16, 16, 32, 64, 100, 256])
    cache = dtype if dtype == "f32" else rng.choice(["bf16", "bf16", "e4m3"])
    if op == APPEND:
        B = _log(rng, 1, 128)
        hi = _log(rng, 1, max(1, min(8192, 350000000 // (B * (Hq + 2 * Hk) * D * SIZE[dtype]))))
        return _append(B, rng.choice([0, 1, hi // 2]) if hi > 1 else 1, hi, Hq, Hk, D, dtype=dtype, cache=cache, page=page,
                       past=rng.choice([0, _log(rng, 1, 5000)]), span=rng.choice([0, 8192]), **rest)
    B = _log(rng, 1, 256)
    row = Hk * D * SIZE[cache]
    hi = _log(rng, 8, max(64, min(200000, 400000000 // (B * row), 30000000 // (B * Hq))))
    lo = rng.choice([0, 1, hi // 2, hi]) if B > 1 else hi
    keep = rng.choice([1.0, 1.0, 0.5, 0.15]) if hi >= 100 else 1.0
    window = rng.choice([0, 0, 0, 1 if keep == 1.0 else 0, _log(rng, 2 if keep == 1.0 else 50, hi + 2)])
    return _attend(B, lo, hi, Hq, Hk, D, dtype=dtype, cache=cache, page=page, heads_first=rest["heads_first"], window=window,
                   keep=keep)


# ------------------------------------------------------------------ inputs
def _lengths(lo, hi, B):
    """B lengths spread evenly from lo to hi, long and short ones mixed: the same for every seed, so that work() knows them."""
    step = 1 + B // 3
    while math.gcd(step, B) != 1:
        step += 1
    return [lo + (hi - lo) * ((b * step + B - 1) % B) // max(1, B - 1) for b in range(B)]


def _visible(c):
    """For each sequence: its first visible key and how many of the keys from there on are kept."""
    got = []
    for n in _lengths(c["lo"], c["hi"], c["B"]):
        first = max(0, n - c["window"]) if c["window"] else 0
        got.append((n, first, n - first if c["keep"] == 1.0 else int(c["keep"] * (n - first))))
    return got


def _frequencies(c):
    """Radians a position, one a rotated pair; stretched contexts turn slow pairs slower still and leave fast ones alone."""
    i = torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64)
    f = 1e6 ** (-2.0 * i / c["rot"])
    turns = 32768.0 / (2 * math.pi) * f  # over the context that the model has seen in training
    blend = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
    return f * (blend + (1 - blend) / c["stretch"])


def _rows(gen, dtype, *shape):
    """Projections as they come out of a matrix product: heads with their own scale, a few strong components."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    x *= torch.exp(0.3 * torch.randn(shape[-2:], generator=gen, device="cuda"))
    return x.to(DTYPES[dtype])


def _pages(gen, B, W):
    """Tables of B sequences over a pool with spare pages, in no order."""
    count = B * W + 3
    return torch.randperm(count, generator=gen, device="cuda")[:B * W].reshape(B, W).to(torch.int32), count


def _pool(gen, c, pages):
    """A cache [pages, page, Hk, D]; heads_first holds a page's heads one after another."""
    shape = (pages, c["Hk"], c["page"], c["D"]) if c["heads_first"] else (pages, c["page"], c["Hk"], c["D"])
    wide = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32 if c["cache"] == "f32" else torch.bfloat16)
    if c["cache"] == "e4m3":
        wide = (wide * 60).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
    return wide.permute(0, 2, 1, 3) if c["heads_first"] else wide


def _scales(gen, c):
    return (0.01 + 0.02 * torch.rand(c["Hk"], generator=gen, device="cuda")) if c["cache"] == "e4m3" else None


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c}
    B, Hq, Hk, D = c["B"], c["Hq"], c["Hk"], c["D"]
    if c["op"] == ROTARY:
        T = c["T"]
        if c["heads_first"]:
            x = [_rows(gen, c["dtype"], B, T, h, D).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for h in (Hq, Hk)]
        else:  # parts of one projection of queries, keys and values
            both = _rows(gen, c["dtype"], B, T, Hq + 2 * Hk, D)
            x = [both[:, :, :Hq], both[:, :, Hq:Hq + Hk]]
        at = torch.rand(B, c["span"], generator=gen, device="cuda").argsort(1)[:, :T] if T > 1 else \
            torch.randint(0, c["span"], (B, T), generator=gen, device="cuda")
        s.update(x=x, pos=at.sort(1).values.contiguous(), freq=_frequencies(c))
        return s
    if c["op"] == APPEND:
        new = _lengths(c["lo"], c["hi"], B)
        past = [c["past"] + 3 * (b % 5) if c["past"] else 0 for b in range(B)]
        W = max(1, -(-max(p + n for p, n in zip(past, new)) // c["page"]))
        T = sum(new)
        table, pages = _pages(gen, B, W)
        both = _rows(gen, c["dtype"], T, Hq + 2 * Hk, D)
        starts = torch.tensor([0] + new, device="cuda", dtype=torch.int32).cumsum(0).to(torch.int32)
        s.update(q=both[:, :Hq], k=both[:, Hq:Hq + Hk], v=both[:, Hq + Hk:], table=table, freq=_frequencies(c),
                 lens=torch.tensor(past, device="cuda", dtype=torch.int32), starts=None if c["lo"] == c["hi"] == 1 else starts,
                 pos=torch.randint(0, c["span"], (T,), generator=gen, device="cuda") if c["span"] else None,
                 k_cache=_pool(gen, c, pages), v_cache=_pool(gen, c, pages), k_scale=_scales(gen, c), v_scale=_scales(gen, c))
        return s
    seen = _visible(c)
    W = max(1, -(-max(n for n, _, _ in seen) // c["page"]))
    table, pages = _pages(gen, B, W)
    lens = torch.tensor([n for n, _, _ in seen], device="cuda", dtype=torch.int32)
    used = torch.arange(W, device="cuda")[None] * c["page"] < lens[:, None]
    s.update(q=_rows(gen, c["dtype"], B, Hq, D), lens=lens, table=torch.where(used, table, -1), k_cache=_pool(gen, c, pages),
             v_cache=_pool(gen, c, pages), k_scale=_scales(gen, c), v_scale=_scales(gen, c), keep=None, ws=None)
    if c["keep"] != 1.0:  # exactly as many kept keys of each sequence as _visible says, at random places of its window
        L = W * c["page"]
        first = torch.tensor([f for _, f, _ in seen], device="cuda")[:, None]
        count = torch.tensor([n for _, _, n in seen], device="cuda")[:, None]
        at = torch.arange(L, device="cuda")[None]
        rank = torch.rand(B, L, generator=gen, device="cuda")
        rank = torch.where((at >= first) & (at < lens[:, None]), rank, 2.0).argsort(1).argsort(1)
        s["keep"] = rank < count
    return s


# ------------------------------------------------------------------ the plain form
def _turned(x, pos, freq, layout, back=False):
    """x [..., heads, D] in 32 bits, rotated at pos [...]. The angle is taken in 64 bits: 32 do not hold a long position's."""
    angle = (pos.double()[..., None] * freq).remainder(2 * math.pi).float()[..., None, :]
    cos, sin = angle.cos(), -angle.sin() if back else angle.sin()
    n = freq.numel()
    x, rest = x[..., :2 * n].float(), x[..., 2 * n:].float()
    if layout == "half":
        a, b = x[..., :n], x[..., n:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., ::2], x[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, rest], -1)


def _stored(x, cache, scale):
    """What the cache holds of x [T, Hk, D], as bytes where it holds 8 bits."""
    if scale is None:
        return x.to(cache.dtype)
    return (x / scale[:, None]).clamp(-LARGEST, LARGEST).to(cache.dtype).view(torch.uint8)


def _plain_append(s):
    c = s["case"]
    T = s["k"].shape[0]
    row = torch.arange(T, device="cuda")
    if s["starts"] is None:
        b, i, new = row, torch.zeros_like(row), torch.ones_like(s["lens"])
    else:
        b = torch.searchsorted(s["starts"][1:].long(), row, right=True)
        i, new = row - s["starts"].long()[b], s["starts"][1:] - s["starts"][:-1]
    slot = s["lens"].long()[b] + i
    page, at = s["table"].long()[b, slot // c["page"]], slot % c["page"]
    pos = slot if s["pos"] is None else s["pos"]
    k = _turned(s["k"], pos, s["freq"], c["layout"])
    for cache, x, scale in ((s["k_cache"], k, s["k_scale"]), (s["v_cache"], s["v"].float(), s["v_scale"])):
        held = cache if scale is None else cache.view(torch.uint8)
        held[page, at] = _stored(x, cache, scale)
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": s["lens"] + new,
            "q": _turned(s["q"], pos, s["freq"], c["layout"]).to(s["q"].dtype)}


def _plain_attend(s):
    c = s["case"]
    B, Hq, Hk, D = c["B"], c["Hq"], c["Hk"], c["D"]
    page = s["table"].long().clamp(min=0)
    L = page.shape[1] * c["page"]

    def rows(cache, scale):
        if scale is None:
            return cache[page].reshape(B, L, Hk, D).float()
        return cache.view(torch.uint8)[page].view(torch.float8_e4m3fn).reshape(B, L, Hk, D).float() * scale[:, None]

    at, lens = torch.arange(L, device="cuda")[None], s["lens"][:, None]
    seen = at < lens
    if c["window"]:
        seen &= at >= lens - c["window"]
    if s["keep"] is not None:
        seen &= s["keep"]
    q = s["q"].float().reshape(B, Hk, Hq // Hk, D)
    score = q @ rows(s["k_cache"], s["k_scale"]).permute(0, 2, 3, 1) / math.sqrt(D)
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (score - top).exp()
    total = p.sum(-1, keepdim=True)
    v = torch.where(seen[:, :, None, None], rows(s["v_cache"], s["v_scale"]), 0.0)
    out = p @ v.permute(0, 2, 1, 3) / torch.where(total == 0, 1.0, total)
    return {"out": out.reshape(B, Hq, D).to(s["q"].dtype), "lse": (total.log() + top).reshape(B, Hq)}


def _plain(s):
    c = s["case"]
    if c["op"] == ROTARY:
        return [_turned(x, s["pos"], s["freq"], c["layout"], c["gradient"]).to(x.dtype) for x in s["x"]]
    return _plain_append(s) if c["op"] == APPEND else _plain_attend(s)


# ------------------------------------------------------------------ the framework's operators
def _framework(s):
    import paper_2608_13226_gb300 as cp
    c = s["case"]
    if c["op"] == ROTARY:
        return cp.coverprune_rotary(s["x"], s["pos"], s["freq"], layout=c["layout"], inverse=c["gradient"])
    if c["op"] == APPEND:
        r = cp.coverprune_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["lens"], starts=s["starts"],
                                       pos=s["pos"], inv_freq=s["freq"], layout=c["layout"], q=s["q"], k_scale=s["k_scale"],
                                       v_scale=s["v_scale"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": r["lens"], "q": r["q"]}
    r = cp.coverprune_decode_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], window=c["window"],
                                       keep=s["keep"], k_scale=s["k_scale"], v_scale=s["v_scale"], lse=True, ws=s["ws"])
    s["ws"] = r["ws"]  # the workspace is kept between calls, as a serving program keeps it
    return {"out": r["out"], "lse": r["lse"]}


def run(state):
    return _framework(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    e, D, Hq, Hk, B = SIZE[c["dtype"]], c["D"], c["Hq"], c["Hk"], c["B"]
    if c["op"] == ROTARY:
        rows = B * c["T"] * (Hq + Hk)
        return {"bytes": rows * D * e * 2 + B * c["T"] * 8, "flops": rows * c["rot"] * 3}
    if c["op"] == APPEND:
        T = sum(_lengths(c["lo"], c["hi"], B))
        held = SIZE[c["cache"]]
        return {"bytes": T * ((2 * Hq + 2 * Hk) * D * e + 2 * Hk * D * held + (8 if c["span"] else 0)) + 12 * B,
                "flops": T * (Hq + Hk) * c["rot"] * 3}
    seen = _visible(c)
    keys, masked = sum(n for _, _, n in seen), sum(n - f for n, f, _ in seen) if c["keep"] != 1.0 else 0
    pages = sum(-(-n // c["page"]) - f // c["page"] for n, f, _ in seen)
    return {"bytes": keys * Hk * D * SIZE[c["cache"]] * 2 + masked + 4 * pages + 4 * B + B * Hq * (2 * D * e + 4),
            "flops": 4 * keys * Hq * D}


# ------------------------------------------------------------------ 64 bits, from the definitions
def _spin(x, pos, c, back=False):
    """The rotation as a product of complex numbers. x [..., heads, D] and pos [...]."""
    x, n = x.double(), c["rot"] // 2
    unit = torch.polar(torch.ones((), device="cuda", dtype=torch.float64), pos.double()[..., None, None] * _frequencies(c))
    unit = unit.conj() if back else unit
    out = x.clone()
    first, second = (slice(0, n), slice(n, 2 * n)) if c["layout"] == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = torch.complex(x[..., first], x[..., second]) * unit
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _held(x, scale):
    """Cached rows [n, D] of one head in 64 bits."""
    return x.double() if scale is None else x.float().double() * float(scale)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == ROTARY:
        return [_spin(x, s["pos"], c, c["gradient"]) for x in s["x"]]
    page = c["page"]
    if c["op"] == APPEND:
        # the cache as it would be without rounding, in its own unit where it holds 8 bits
        k_cache, v_cache = s["k_cache"].float().double(), s["v_cache"].float().double()
        past, table = s["lens"].tolist(), s["table"].tolist()
        starts = list(range(c["B"] + 1)) if s["starts"] is None else s["starts"].tolist()
        one = torch.ones(c["Hk"], device="cuda", dtype=torch.float64)
        k_one = one if s["k_scale"] is None else s["k_scale"].double()
        v_one = one if s["v_scale"] is None else s["v_scale"].double()
        pos = s["pos"] if s["pos"] is not None else torch.tensor(
            [past[b] + i for b in range(c["B"]) for i in range(starts[b + 1] - starts[b])], device="cuda", dtype=torch.int64)
        k, v = _spin(s["k"], pos, c) / k_one[:, None], s["v"].double() / v_one[:, None]
        if c["cache"] == "e4m3":
            k, v = k.clamp(-LARGEST, LARGEST), v.clamp(-LARGEST, LARGEST)
        for b in range(c["B"]):
            lo, n = past[b], starts[b + 1] - starts[b]
            for j in range(lo // page, -(-(lo + n) // page)):  # the part of each page that the new rows fill
                u, w = max(lo, j * page), min(lo + n, (j + 1) * page)
                to, of = slice(u - j * page, w - j * page), slice(starts[b] + u - lo, starts[b] + w - lo)
                k_cache[table[b][j], to], v_cache[table[b][j], to] = k[of], v[of]
        return {"k_cache": k_cache, "v_cache": v_cache, "lens": None, "q": _spin(s["q"], pos, c)}
    G = c["Hq"] // c["Hk"]
    out = torch.zeros(c["B"], c["Hq"], c["D"], device="cuda", dtype=torch.float64)
    lse = torch.full((c["B"], c["Hq"]), -math.inf, device="cuda", dtype=torch.float64)
    table = s["table"].long()
    for b, (n, first, _) in enumerate(_visible(c)):
        key = torch.arange(first, n, device="cuda")
        if s["keep"] is not None:
            key = key[s["keep"][b, first:n]]
        if not key.numel():
            continue
        at = (table[b, key // page], key % page)
        for h in range(c["Hk"]):
            heads = slice(h * G, (h + 1) * G)
            k, v = (_held(s[p + "_cache"][:, :, h].float()[at] if c["cache"] != "e4m3" else
                          s[p + "_cache"].view(torch.uint8)[:, :, h][at].view(torch.float8_e4m3fn),
                          None if s[p + "_scale"] is None else s[p + "_scale"][h]) for p in ("k", "v"))
            score = s["q"][b, heads].double() @ k.T / math.sqrt(c["D"])
            lse[b, heads] = score.logsumexp(-1)
            out[b, heads] = (score - lse[b, heads, None]).exp() @ v
    return {"out": out, "lse": lse}
