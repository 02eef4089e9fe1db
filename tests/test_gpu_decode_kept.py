"""The decoding example: one layer on the kept tokens of pruned scenes against the
same layer in 64 bits over the kept tokens alone."""
import pytest
import torch

import paper_2608_13226_gb300 as cp
from paper_2608_13226_gb300 import decode_kept as dk
from gpu_util import batch_to_dev, scene

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_13226_gb300 import build
    build.build()
    cp.load()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_layer_on_kept_tokens(dtype):
    f, pos, fr = batch_to_dev([scene("long_video", i, N=700, D=256) for i in range(3)])
    kept = cp.coverprune_select(f, pos, fr, 90)["kept"]
    rows = cp.coverprune_gather(f, pos, fr, kept)[0]
    layer = dk.make_layer(256, 14, 2, width=64, context=4.0)
    cache = dk.Cache(layer, 3, 100, dtype)
    dk.fill(layer, cache, rows, kept)
    assert cache.lens.tolist() == [90] * 3
    x = f[:, 5].contiguous()
    at = torch.tensor([700, 701, 5000], device="cuda")
    got = dk.step(layer, cache, x, at).double()
    assert cache.lens.tolist() == [91] * 3 and int(cache.status) == 0

    def turn(t, p):  # [n, heads, width] at p [n]
        a = p.double()[:, None, None] * layer.freq
        u, w = t.double().chunk(2, -1)
        return torch.cat([u * a.cos() - w * a.sin(), w * a.cos() + u * a.sin()], -1)

    half = {torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}[dtype]  # half a unit of what the cache holds
    for b in range(3):
        q, k, v = layer.project(torch.cat([rows[b], x[b:b + 1]]))
        p = torch.cat([kept[b], at[b:b + 1]])
        q, k, v = turn(q[-1:], p[-1:])[0], turn(k, p), v.double()
        k, v = k.repeat_interleave(7, 1), v.repeat_interleave(7, 1)
        s = torch.einsum("hd,jhd->hj", q, k) / 8
        w = s.softmax(-1)
        o = torch.einsum("hj,jhd->hd", w, v)
        want = o.reshape(1, -1) @ layer.out.double()
        # queries (2^-8) and keys and values (half, and for 8 bits 2^-10 of the scale below
        # 2^-6 of it) are rounded: scores are off by d, weights by 2 d, outputs by that and
        # half of |v|, then rounded to 2^-8, and once more after the projection
        low = 0.05 * 2.0 ** -10 if dtype != torch.bfloat16 else 0.0
        mag = torch.einsum("hd,jhd->hj", q.abs(), k.abs()) / 8
        d = ((half + 2.0 ** -8) * mag + low * q.abs().sum(-1, keepdim=True) / 8).amax(-1, keepdim=True)
        off = torch.einsum("hj,jhd->hd", w, v.abs()) * (2 * d + half + 2.0 ** -7) + low
        tol = off.reshape(1, -1) @ layer.out.double().abs() + 2.0 ** -8 * want.abs() + 256 * 2.0 ** -24
        assert bool(((got[b] - want[0]).abs() <= tol[0]).all())


def test_steps_and_command(capsys):
    """Several steps run on, the cache grows by one key a step, and the command prints both caches."""
    f, pos, fr = batch_to_dev([scene("long_video", i, N=300, D=256) for i in range(2)])
    layer = dk.make_layer(256, 8, 4, width=64)
    cache = dk.Cache(layer, 2, 320)
    dk.fill(layer, cache, f, torch.arange(300, device="cuda").expand(2, 300).contiguous())
    out = dk.decode(layer, cache, f[:, 0].contiguous(), torch.full((2,), 300, device="cuda"), 20)
    assert cache.lens.tolist() == [320] * 2 and bool(out.isfinite().all()) and int(cache.status) == 0
    dk.step(layer, cache, f[:, 1].contiguous(), torch.full((2,), 320, device="cuda"))  # the cache is full
    assert int(cache.status) == cp.CP_EINVAL and cache.lens.tolist() == [320] * 2
    dk.main(["--scenes", "1", "--steps", "2"])
    lines = capsys.readouterr().out.strip().split("\n")
    assert len(lines) == 2 and lines[0].startswith("kept") and lines[1].startswith("all")
