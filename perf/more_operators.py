"""The calls of a program that decodes on pruned scenes for a long time and keeps the cache small while it does: keys and values
held in 4 bits, attention over such a cache, attention that adds up what weight each cached key got, and the eviction of
the lightest keys.

A case names one operator ("op"), its sizes and the options that the program would set.  `own` picks what `run` does: the
framework's entry points, or the same operators in elementary torch operations.  Heads are those of the feature widths
of the pruned scenes (3584 = 28 x 128, 1280 = 20 x 64, 256 = 4 x 64), lengths those of pruned and unpruned scenes (1229 and
8192 tokens) with some text, and longer caches.

4 bits: 16 components of a row share a scale s of 8 bits (e4m3), and a component is a whole number n from -7 to 7 that
stands for n s (times the head's own scale, if it has one).  A byte holds n + 8 of two components, the first in its low half.
"""
import math

import torch

own = False

KEEP, ATTEND, WEIGH, EVICT = "keep", "attend", "weigh", "evict"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}
LARGEST = 448.0  # the largest e4m3 value
BLOCK = 16       # components of a scale


def _keep(B, lo, hi, Hq, Hk, D, **options):
    c = {"op": KEEP, "B": B, "lo": lo, "hi": hi, "past": 0, "Hq": Hq, "Hk": Hk, "D": D, "rot": 0, "layout": "half",
         "dtype": "bf16", "cache": "4 bits", "page": 16, "heads_first": False, "scaled": False}
    c.update(options)
    return c


def _attend(B, lo, hi, Hq, Hk, D, **options):
    c = {"op": ATTEND, "B": B, "lo": lo, "hi": hi, "Hq": Hq, "Hk": Hk, "D": D, "dtype": "bf16", "cache": "4 bits", "page": 16,
         "heads_first": False, "window": 0, "keep": 1.0, "scaled": False}
    c.update(options)
    return c


def _weigh(B, lo, hi, Hq, Hk, D, **options):
    return dict(_attend(B, lo, hi, Hq, Hk, D, **{"cache": "bf16", **options}), op=WEIGH)


def _evict(B, lo, hi, Hk, D, left, **options):
    c = {"op": EVICT, "B": B, "lo": lo, "hi": hi, "Hk": Hk, "D": D, "left": left, "first": 4, "recent": min(64, left // 4),
         "cache": "bf16", "page": 16, "heads_first": False}
    c.update(options)
    return c


def listed():
    return [
        # the prompt of the throughput batch on its way into 4 bits, keys turned before; read back for the prompt's own attention
        dict(_keep(32, 900, 1500, 0, 4, 128), name="keep prompt"),
        # one token of each of 64 sequences, key and queries turned on the way: what every decoded token pays in every layer
        dict(_keep(64, 1, 1, 28, 4, 128, past=1229, rot=128, heads_first=True, page=32), name="keep token"),
        # ragged prompts of a small model in 32 bits, empty ones among them, narrow rows, a scale a head, pages of 7
        dict(_keep(21, 0, 3001, 0, 6, 96, dtype="f32", page=7, scaled=True), name="keep ragged f32"),
        # one scene alone after pruning, some text in: the latency between two words
        dict(_attend(1, 1500, 1500, 28, 4, 128), name="attend one scene"),
        # the throughput batch unpruned
        dict(_attend(32, 8192, 8704, 28, 4, 128), name="attend batch"),
        # many sequences of very different lengths, heads before slots in a page, a scale a head
        dict(_attend(128, 500, 16000, 16, 2, 128, page=32, heads_first=True, scaled=True), name="attend ragged"),
        # one scene again, its keys' weights added up for a later eviction
        dict(_weigh(1, 1500, 1500, 28, 4, 128), name="weigh one scene"),
        # the throughput batch after pruning to 15%
        dict(_weigh(32, 1229, 1741, 28, 4, 128), name="weigh batch kept"),
        # long scenes in 4 bits, narrow heads, half of the keys marked
        dict(_weigh(16, 8192, 8704, 20, 20, 64, cache="4 bits", keep=0.5), name="weigh 4 bits marked"),
        # sequences a few tokens over what they may hold, as after some steps of decoding: latency
        dict(_evict(64, 1237, 1245, 4, 128, 1229, cache="e4m3", heads_first=True, page=32), name="evict few"),
        # unpruned scenes cut to 15% once their question has been read
        dict(_evict(32, 8192, 8704, 4, 128, 1229), name="evict batch"),
        # one very long cache, halved
        dict(_evict(1, 200001, 200001, 8, 128, 100000, page=64), name="evict long"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice([KEEP, ATTEND, ATTEND, WEIGH, WEIGH, EVICT])
    page = rng.choice([1, 7, 16, 16, 32, 64, 100, 256])
    first = rng.random() < 0.3
    cache = "4 bits" if op in (KEEP, ATTEND) else rng.choice(["bf16", "bf16", "e4m3", "f32", "4 bits"])
    if op == EVICT and cache == "4 bits":
        cache = "bf16"  # such rows are moved as bytes, as any others
    D = rng.choice([32, 64, 64, 96, 128, 128, 128, 256] if cache == "4 bits" else [64, 80, 96, 128, 128, 256])
    Hk = rng.choice([1, 2, 3, 4, 8])
    Hq = Hk * rng.choice([1, 2, 4, 5, 7, 8, 12, 16])
    if op == KEEP:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        B = _log(rng, 1, 128)
        hi = _log(rng, 1, max(1, min(8192, 80000000 // (B * Hk * D * SIZE[dtype]))))
        # A turned key is known to 32 bits and may lie next to a border between two numbers: few are turned here
        turned = dtype == "bf16" and B * hi * Hk * D <= 50000
        return _keep(B, rng.choice([0, 1, hi // 2]) if hi > 1 else 1, hi, Hq if turned else 0, Hk, D, dtype=dtype, page=page,
                     past=rng.choice([0, _log(rng, 1, 5000)]), rot=rng.choice([D, D // 2, D // 4]) if turned else 0,
                     layout=rng.choice(["half", "interleaved"]), heads_first=first, scaled=rng.random() < 0.5)
    if op == EVICT:
        B = _log(rng, 1, 128)
        row = 2 * Hk * D * SIZE[cache]
        hi = _log(rng, 8, max(64, min(200000, 800000000 // (B * row))))
        left = max(1, int(hi * rng.choice([0.05, 0.15, 0.5, 0.9, 0.99])))
        return _evict(B, rng.choice([0, 1, hi // 2, hi]) if B > 1 else hi, hi, Hk, D, left, first=rng.choice([0, min(4, left // 2)]),
                      recent=rng.choice([0, min(64, left // 4), left // 2]), cache=cache, page=page, heads_first=first)
    B = _log(rng, 1, 256)
    row = Hk * D * SIZE.get(cache, 0.5625)
    hi = _log(rng, 8, max(64, int(min(200000, 200000000 // (B * row), 400000000 // (B * Hk * D), 30000000 // (B * Hq)))))
    lo = rng.choice([0, 1, hi // 2, hi]) if B > 1 else hi
    keep = rng.choice([1.0, 1.0, 0.5, 0.15]) if hi >= 100 else 1.0
    window = rng.choice([0, 0, 0, 1 if keep == 1.0 else 0, _log(rng, 2 if keep == 1.0 else 50, hi + 2)])
    return (_attend if op == ATTEND else _weigh)(B, lo, hi, Hq, Hk, D, dtype="f32" if cache == "f32" else "bf16", cache=cache,
                                                 page=page, heads_first=first, window=window, keep=keep,
                                                 scaled=cache == "4 bits" and rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _lengths(lo, hi, B):
    """B lengths spread evenly from lo to hi, long and short ones mixed: the same for every seed, so that work() knows them."""
    step = 1 + B // 3
    while math.gcd(step, B) != 1:
        step += 1
    return [lo + (hi - lo) * ((b * step + B - 1) % B) // max(1, B - 1) for b in range(B)]


def _visible(c):
    """For each sequence: its length, its first visible key and how many of the keys from there on are marked."""
    got = []
    for n in _lengths(c["lo"], c["hi"], c["B"]):
        first = max(0, n - c["window"]) if c["window"] else 0
        got.append((n, first, n - first if c["keep"] == 1.0 else int(c["keep"] * (n - first))))
    return got


def _frequencies(c):
    i = torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64)
    return 1e6 ** (-2.0 * i / c["rot"])


def _rows(gen, dtype, *shape):
    """Projections as they come out of a matrix product: heads with their own scale, a few strong components."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    x *= torch.exp(0.3 * torch.randn(shape[-2:], generator=gen, device="cuda"))
    return x.to(DTYPES[dtype])


def _pages(gen, B, W):
    """Tables of B sequences over a pool with spare pages, in no order."""
    count = B * W + 3
    return torch.randperm(count, generator=gen, device="cuda")[:B * W].reshape(B, W).to(torch.int32), count


def _blocks_of(c):
    """Bytes of a row's scales: one for 16 components, in fours."""
    return -(-c["D"] // (4 * BLOCK)) * 4


def _pool(gen, c, pages):
    """A cache [pages, page, Hk, D] and, in 4 bits, its scales; heads_first holds a page's heads one after another."""
    def shaped(x):
        return x.permute(0, 2, 1, 3) if c["heads_first"] else x

    def shape(n):
        return (pages, c["Hk"], c["page"], n) if c["heads_first"] else (pages, c["page"], c["Hk"], n)

    if c["cache"] == "4 bits":
        # whole numbers as rows of a normal distribution give them: two bell-shaped halves of a byte from 1 to 15
        bell = (torch.randn(4096, generator=gen, device="cuda") * 2.5).round().clamp(-7, 7).to(torch.int32) + 8
        bytes_ = (bell[:2048] | bell[2048:] << 4).to(torch.uint8)
        held = torch.randint(0, 2048, shape(c["D"] // 2), generator=gen, device="cuda", dtype=torch.int16)
        scale = 0.15 + 0.3 * torch.rand(shape(_blocks_of(c)), generator=gen, device="cuda")
        scale[..., c["D"] // BLOCK:] = 0.0
        return shaped(bytes_[held.int()]), shaped(scale.to(torch.float8_e4m3fn))
    x = torch.randn(shape(c["D"]), generator=gen, device="cuda", dtype=torch.float32 if c["cache"] == "f32" else torch.bfloat16)
    if c["cache"] == "e4m3":
        x = (x * 60).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
    return shaped(x), None


def _scales(gen, c):
    """A factor a head: an 8-bit cache has one always, a 4-bit one where the case says so."""
    if c["cache"] == "e4m3" and c["op"] != EVICT:
        return 0.01 + 0.02 * torch.rand(c["Hk"], generator=gen, device="cuda")
    return 0.5 + torch.rand(c["Hk"], generator=gen, device="cuda") if c.get("scaled") else None


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c}
    B, Hk, D = c["B"], c["Hk"], c["D"]
    if c["op"] == KEEP:
        new = _lengths(c["lo"], c["hi"], B)
        past = [c["past"] + 3 * (b % 5) if c["past"] else 0 for b in range(B)]
        W = max(1, -(-max(p + n for p, n in zip(past, new)) // c["page"]))
        T, Hq = sum(new), c["Hq"]
        table, pages = _pages(gen, B, W)
        both = _rows(gen, c["dtype"], T, Hq + 2 * Hk, D)  # parts of one projection of queries, keys and values
        starts = torch.tensor([0] + new, device="cuda", dtype=torch.int32).cumsum(0).to(torch.int32)
        s.update(q=both[:, :Hq] if Hq else None, k=both[:, Hq:Hq + Hk], v=both[:, Hq + Hk:], table=table,
                 freq=_frequencies(c) if c["rot"] else None, lens=torch.tensor(past, device="cuda", dtype=torch.int32),
                 starts=None if c["lo"] == c["hi"] == 1 else starts, k_scale=_scales(gen, c), v_scale=_scales(gen, c))
        s["k_cache"], s["k_block"] = _pool(gen, c, pages)
        s["v_cache"], s["v_block"] = _pool(gen, c, pages)
        return s
    lens = _lengths(c["lo"], c["hi"], B)
    W = max(1, -(-max(lens) // c["page"]))
    L = W * c["page"]
    table, pages = _pages(gen, B, W)
    s["lens"] = torch.tensor(lens, device="cuda", dtype=torch.int32)
    s["table"] = torch.where(torch.arange(W, device="cuda")[None] * c["page"] < s["lens"][:, None], table, -1)
    s["k_cache"], s["k_block"] = _pool(gen, c, pages)
    s["v_cache"], s["v_block"] = _pool(gen, c, pages)
    at = torch.arange(L, device="cuda")[None]
    if c["op"] != ATTEND:  # weights so far: some keys have got much, most little, some nothing; 0 behind a sequence's end
        w = torch.exp(2.0 * torch.randn(B, L, generator=gen, device="cuda")) * (torch.rand(B, L, generator=gen, device="cuda") > 0.1)
        if c["op"] == WEIGH:  # about what one token before gave them
            w *= c["Hq"] / (7.0 * s["lens"].clamp(min=1)[:, None])
        s["weight"] = torch.where(at < s["lens"][:, None], w, 0.0)
    if c["op"] == EVICT:
        return s
    s.update(q=_rows(gen, c["dtype"], B, c["Hq"], D), k_scale=_scales(gen, c), v_scale=_scales(gen, c), keep=None, ws=None)
    if c["keep"] != 1.0:  # exactly as many marked keys of each sequence as _visible says, at random places of its window
        seen = _visible(c)
        first = torch.tensor([f for _, f, _ in seen], device="cuda")[:, None]
        count = torch.tensor([n for _, _, n in seen], device="cuda")[:, None]
        rank = torch.rand(B, L, generator=gen, device="cuda")
        rank = torch.where((at >= first) & (at < s["lens"][:, None]), rank, 2.0).argsort(1).argsort(1)
        s["keep"] = rank < count
    return s


# ------------------------------------------------------------------ the plain form
def _turned(x, pos, freq, layout):
    """x [..., heads, D] in 32 bits, rotated at pos [...]. The angle is taken in 64 bits: 32 do not hold a long position's."""
    x = x.float()
    if freq is None:
        return x
    angle = (pos.double()[..., None] * freq).remainder(2 * math.pi)[..., None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    n = freq.numel()
    x, rest = x[..., :2 * n], x[..., 2 * n:]
    if layout == "half":
        a, b = x[..., :n], x[..., n:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., ::2], x[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, rest], -1)


def _fours(x, scale):
    """Rows x [T, Hk, D] in 32 bits as bytes of two components, and their scales."""
    x = x.unflatten(-1, (-1, BLOCK))
    head = torch.ones((), device="cuda") if scale is None else scale[:, None]
    s = (x.abs().amax(-1) / (7.0 * head)).clamp(max=LARGEST).to(torch.float8_e4m3fn)
    step = (s.float() * head)[..., None]
    n = torch.where(step == 0, 0.0, x / torch.where(step == 0, 1.0, step)).round().clamp(-7, 7).to(torch.int32).flatten(-2) + 8
    return (n[..., ::2] | n[..., 1::2] << 4).to(torch.uint8), s


def _values(held, blocks, scale, D):
    """What bytes [..., D / 2] with scales [..., >= D / 16] stand for, in 32 bits."""
    n = torch.stack([held & 15, held >> 4], -1).flatten(-2).float() - 8.0
    x = n * blocks[..., :D // BLOCK].float().repeat_interleave(BLOCK, -1)
    return x if scale is None else x * scale[:, None]


def _plain_keep(s):
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
    got = {"lens": s["lens"] + new, "q": None if s["q"] is None else _turned(s["q"], slot, s["freq"], c["layout"]).to(s["q"].dtype)}
    n = c["D"] // BLOCK
    for p, x in (("k", _turned(s["k"], slot, s["freq"], c["layout"])), ("v", s["v"].float())):
        held, blocks = _fours(x, s[p + "_scale"])
        s[p + "_cache"][page, at] = held
        s[p + "_block"].view(torch.uint8)[..., :n][page, at] = blocks.view(torch.uint8)
        blocks = s[p + "_block"].view(torch.uint8)[page, at].view(torch.float8_e4m3fn)
        got[p] = _values(s[p + "_cache"][page, at], blocks, s[p + "_scale"], c["D"]).bfloat16()
    return got


def _plain_attend(s):
    c = s["case"]
    B, Hq, Hk, D = c["B"], c["Hq"], c["Hk"], c["D"]
    page = s["table"].long().clamp(min=0)
    L = page.shape[1] * c["page"]

    def rows(p):
        cache, scale = s[p + "_cache"], s[p + "_scale"]
        if c["cache"] == "4 bits":
            return _values(cache[page], s[p + "_block"].view(torch.uint8)[page].view(torch.float8_e4m3fn), scale, D).reshape(B, L, Hk, D)
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
    score = q @ rows("k").permute(0, 2, 3, 1) / math.sqrt(D)
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (score - top).exp()
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    v = torch.where(seen[:, :, None, None], rows("v"), 0.0)
    got = {"out": (p @ v.permute(0, 2, 1, 3)).reshape(B, Hq, D).to(s["q"].dtype), "lse": (total.log() + top).reshape(B, Hq)}
    if c["op"] == WEIGH:
        s["weight"] += p.sum((1, 2))
        got["weight"] = s["weight"]
    return got


def _plain_evict(s):
    c = s["case"]
    L, n = s["weight"].shape[1], c["left"]
    at, lens = torch.arange(L, device="cuda")[None], s["lens"].long()[:, None]
    # what stays in any case comes first, then by weight, the earlier of equals first; what is not there comes last
    rank = torch.where((at < c["first"]) | (at >= lens - c["recent"]), math.inf, s["weight"])
    rank = torch.where(at < lens, rank, -math.inf)
    order = torch.argsort(rank, dim=1, descending=True, stable=True)[:, :n]
    left = torch.minimum(lens, torch.full_like(lens, n))
    to = torch.arange(order.shape[1], device="cuda")[None]
    kept = torch.where(to < left, order, L).sort(1).values
    b, i = (to < left).nonzero(as_tuple=True)
    j = kept[b, i]
    table = s["table"].long()
    src, dst = (table[b, j // c["page"]], j % c["page"]), (table[b, i // c["page"]], i % c["page"])
    for p in ("k_cache", "v_cache"):
        x = s[p].view(torch.uint8) if c["cache"] == "e4m3" else s[p]
        x[dst] = x[src]
    weight = torch.zeros_like(s["weight"])
    weight[b, i] = s["weight"][b, j]
    held = torch.full((c["B"], n), -1, device="cuda", dtype=torch.int32)
    held[b, i] = j.to(torch.int32)
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": left[:, 0].to(torch.int32), "weight": weight, "kept": held}


def _plain(s):
    op = s["case"]["op"]
    return _plain_keep(s) if op == KEEP else _plain_evict(s) if op == EVICT else _plain_attend(s)


# ------------------------------------------------------------------ the framework's operators
def _framework(s):
    import paper_2608_13226_gb300 as cp
    c = s["case"]
    if c["op"] == KEEP:
        how = {"starts": s["starts"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "k_block": s["k_block"], "v_block": s["v_block"]}
        r = cp.coverprune_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["lens"], inv_freq=s["freq"],
                                       layout=c["layout"], q=s["q"], **how)
        # the rows that were just written, as attention will see them
        k, v = cp.coverprune_cache_read(s["k_cache"], s["v_cache"], s["table"], s["lens"], tokens=s["k"].shape[0],
                                        **how)
        return {"lens": r["lens"], "q": r["q"], "k": k, "v": v}
    if c["op"] == EVICT:
        r = cp.coverprune_cache_evict(s["k_cache"], s["v_cache"], s["table"], s["lens"], s["weight"], c["left"], first=c["first"],
                                      recent=c["recent"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": r["lens"], "weight": r["weight"], "kept": r["kept"]}
    r = cp.coverprune_decode_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], window=c["window"],
                                       keep=s["keep"], k_scale=s["k_scale"], v_scale=s["v_scale"], k_block=s["k_block"],
                                       v_block=s["v_block"], weight=s.get("weight"), lse=True, ws=s["ws"])
    s["ws"] = r["ws"]  # the workspace is kept between calls, as a serving program keeps it
    return {"out": r["out"], "lse": r["lse"], **({"weight": s["weight"]} if c["op"] == WEIGH else {})}


def run(state):
    return _framework(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def _row_bytes(c):
    """Bytes of a cached row of one head."""
    return c["D"] // 2 + c["D"] // BLOCK if c["cache"] == "4 bits" else c["D"] * SIZE[c["cache"]]


def work(case):
    c = case
    D, Hk, B = c["D"], c["Hk"], c["B"]
    lens = _lengths(c["lo"], c["hi"], B)
    if c["op"] == KEEP:
        T, e = sum(lens), SIZE[c["dtype"]]
        # rows in, into the cache, and out again in bfloat16 as the cache has them; queries in and out
        return {"bytes": T * (2 * Hk * (D * e + 2 * D + _row_bytes(c)) + 2 * c["Hq"] * D * e) + 12 * B,
                "flops": T * (2 * Hk * D * 6 + (c["Hq"] + Hk) * c["rot"] * 3)}
    if c["op"] == EVICT:
        # rows that go from where they are to their new place; weights in and out
        moved = sum(min(n, c["left"]) - c["first"] for n in lens if n > c["left"])
        return {"bytes": moved * 2 * 2 * Hk * _row_bytes(c) + 4 * sum(lens) + 8 * B * c["left"] + 8 * B, "flops": 4 * sum(lens)}
    seen = _visible(c)
    keys, looked = sum(n for _, _, n in seen), sum(n - f for n, f, _ in seen) if c["keep"] != 1.0 else 0
    pages = sum(-(-n // c["page"]) - f // c["page"] for n, f, _ in seen)
    return {"bytes": keys * (Hk * _row_bytes(c) * 2 + (8 if c["op"] == WEIGH else 0)) + looked + 4 * pages + 4 * B +
            B * c["Hq"] * (2 * D * SIZE[c["dtype"]] + 4), "flops": 4 * keys * c["Hq"] * D}


# ------------------------------------------------------------------ 64 bits, from the definitions
def _spin(x, pos, c):
    """The rotation as a product of complex numbers. x [..., heads, D] and pos [...]."""
    x, n = x.double(), c["rot"] // 2
    if not n:
        return x
    unit = torch.polar(torch.ones((), device="cuda", dtype=torch.float64), pos.double()[..., None, None] * _frequencies(c))
    out = x.clone()
    first, second = (slice(0, n), slice(n, 2 * n)) if c["layout"] == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = torch.complex(x[..., first], x[..., second]) * unit
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _head(s, p, h, at, c):
    """Cached rows [n, D] of one head at (pages, slots), in 64 bits."""
    x = s[p + "_cache"][:, :, h] if c["cache"] != "e4m3" else s[p + "_cache"].view(torch.uint8)[:, :, h]
    x = x[at]
    if c["cache"] == "4 bits":
        y = torch.empty(x.shape[0], c["D"], device="cuda", dtype=torch.float64)
        y[:, 0::2], y[:, 1::2] = (x % 16).double() - 8, (x // 16).double() - 8
        unit = s[p + "_block"].view(torch.uint8)[:, :, h][at].view(torch.float8_e4m3fn).float().double()
        x = (y.reshape(len(y), -1, BLOCK) * unit[:, :c["D"] // BLOCK, None]).reshape(len(y), -1)
    elif c["cache"] == "e4m3":
        x = x.view(torch.float8_e4m3fn).float()
    return x.double() if s[p + "_scale"] is None else x.double() * float(s[p + "_scale"][h])


def _nearest(x, scale):
    """The value in 4 bits that is nearest to each component of x [T, Hk, D], once a block's largest has set its scale."""
    head = 1.0 if scale is None else scale.double()[:, None, None]
    x = x.reshape(*x.shape[:2], -1, BLOCK)
    most = x.abs().max(-1, keepdim=True).values
    unit = (most / (7 * head)).clamp(max=LARGEST).float().to(torch.float8_e4m3fn).double() * head
    n = torch.where(unit > 0, x / unit, 0.0)
    return (torch.round(n).clamp(-7, 7) * unit).flatten(2)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == KEEP:
        past = s["lens"].tolist()
        starts = list(range(c["B"] + 1)) if s["starts"] is None else s["starts"].tolist()
        pos = torch.tensor([past[b] + i for b in range(c["B"]) for i in range(starts[b + 1] - starts[b])], device="cuda",
                           dtype=torch.int64)
        return {"lens": None, "q": None if s["q"] is None else _spin(s["q"], pos, c),
                "k": _nearest(_spin(s["k"], pos, c), s["k_scale"]), "v": _nearest(s["v"].double(), s["v_scale"])}
    if c["op"] == EVICT:
        return None  # nothing is computed: rows move as they are
    B, Hq, D, G = c["B"], c["Hq"], c["D"], c["Hq"] // c["Hk"]
    if B * c["Hk"] > 1100:
        return None  # a head of a sequence at a time: over 20 seconds
    out = torch.zeros(B, Hq, D, device="cuda", dtype=torch.float64)
    lse = torch.full((B, Hq), -math.inf, device="cuda", dtype=torch.float64)
    weight = s["weight"].double() if c["op"] == WEIGH else None
    table = s["table"].long()
    for b, (n, first, _) in enumerate(_visible(c)):
        key = torch.arange(first, n, device="cuda")
        if s["keep"] is not None:
            key = key[s["keep"][b, first:n]]
        if not key.numel():
            continue
        at = (table[b, key // c["page"]], key % c["page"])
        for h in range(c["Hk"]):
            heads = slice(h * G, (h + 1) * G)
            k, v = _head(s, "k", h, at, c), _head(s, "v", h, at, c)
            score = s["q"][b, heads].double() @ k.T / math.sqrt(D)
            lse[b, heads] = score.logsumexp(-1)
            p = (score - lse[b, heads, None]).exp()
            out[b, heads] = p @ v
            if weight is not None:
                weight[b, key] += p.sum(0)
    return {"out": out, "lse": lse, **({"weight": weight} if weight is not None else {})}
