"""Host side of the decoding model's operators: the rotary frequencies against
their formulas, and the arguments that the entry points refuse before anything
is launched (fake pointers, never dereferenced)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2608_13226_gb300 as cp
from paper_2608_13226_gb300 import binding

FAKE = 0x100000
P = C.c_void_p
TWO = C.c_int64 * 2


@pytest.fixture(scope="module")
def lib():
    from paper_2608_13226_gb300 import build
    build.build()
    return cp.load()


def freq(rot, base=10000.0, **kw):
    return cp.coverprune_rotary_frequencies(rot, base, device="cpu", **kw).numpy()


# the library raises base to -2 i / rot in float64: a few roundings
CLOSE = dict(rtol=1e-13, atol=0)


@pytest.mark.parametrize("rot", [2, 6, 64, 128, 250])
def test_frequencies_plain_linear_base(lib, rot):
    i = np.arange(rot // 2)
    f = 10000.0 ** (-2.0 * i / rot)
    assert freq(rot)[0] == 1.0
    np.testing.assert_allclose(freq(rot), f, **CLOSE)
    np.testing.assert_allclose(freq(rot, stretch="linear", factor=4.0), f / 4, **CLOSE)
    if rot > 2:
        b = freq(rot, stretch="base", factor=8.0)
        assert b[0] == 1.0
        # the slowest pair is factor times slower: base^(-(rot-2)/rot) / 8
        np.testing.assert_allclose(b[-1], f[-1] / 8, rtol=1e-12)


@pytest.mark.parametrize("factor", [1.0, 2.0, 32.0])
def test_frequencies_by_turns(lib, factor):
    rot, L, low, high = 128, 8192.0, 1.0, 4.0
    f = 500000.0 ** (-2.0 * np.arange(64) / rot)
    got = freq(rot, 500000.0, stretch="turns", factor=factor, original=L, low=low, high=high)
    r = L * f / (2 * math.pi)
    np.testing.assert_allclose(got[r >= high], f[r >= high], **CLOSE)
    np.testing.assert_allclose(got[r <= low], f[r <= low] / factor, **CLOSE)
    mid = (r > low) & (r < high)
    assert mid.any()
    w = (r[mid] - low) / (high - low)
    np.testing.assert_allclose(got[mid], f[mid] * (w + (1 - w) / factor), rtol=1e-12)
    assert np.all(np.diff(got) < 0)


def test_frequencies_by_index(lib):
    rot, L, s = 64, 4096.0, 16.0
    f = 10000.0 ** (-2.0 * np.arange(32) / rot)
    got = freq(rot, stretch="index", factor=s, original=L, low=1.0, high=32.0)
    at = lambda t: rot * math.log(L / (2 * math.pi * t)) / (2 * math.log(10000.0))
    lo, hi = math.floor(at(32.0)), math.ceil(at(1.0))
    assert 0 < lo < hi < rot // 2
    w = np.clip((np.arange(32) - lo) / (hi - lo), 0, 1)
    np.testing.assert_allclose(got, f * (1 - w) + f / s * w, rtol=1e-12)


@pytest.mark.parametrize("bad", [dict(rot=0), dict(rot=7), dict(rot=-2), dict(base=1.0), dict(base=float("inf")),
                                 dict(stretch=9), dict(stretch=1, factor=0.5), dict(stretch=1, factor=float("nan")),
                                 dict(stretch=2, rot=2, factor=2.0), dict(stretch=3, factor=2.0),
                                 dict(stretch=3, factor=2.0, original=100.0, low=4.0, high=4.0),
                                 dict(stretch=4, factor=2.0, original=100.0, low=0.0, high=4.0),
                                 dict(stretch=4, factor=2.0, original=-1.0, low=1.0, high=4.0)])
def test_frequencies_refuse(lib, bad):
    a = dict(rot=8, base=10000.0, stretch=0, factor=1.0, original=0.0, low=1.0, high=32.0)
    a.update(bad)
    out = (C.c_double * 8)()
    assert lib.coverprune_rotary_frequencies(*a.values(), out) == cp.CP_EINVAL
    with pytest.raises((cp.CoverPruneError, ValueError)):
        cp.coverprune_rotary_frequencies(8, stretch="other", device="cpu")


def rope(**kw):
    r = binding._Rope(FAKE, 64, 0, 1.0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def rows(**kw):
    r = binding._Rows(FAKE, FAKE, 4, (0, 512, 128), (0, 512, 128))
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def cache(**kw):
    c = binding._Cache(C.sizeof(binding._Cache), cp.CP_BF16, FAKE, FAKE, 10, 16, 4, 128, 16 * 512, 512, 128,
                       None, None, FAKE, 8, 8)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _rotary(lib, r=None, n=1, dt=1, B=0, T=10, D=128, pos=FAKE, rp=None, inverse=0):
    return lib.coverprune_rotary(C.byref(r or rows()), n, dt, B, T, D, P(pos), 0, C.byref(rp or rope()), inverse, None)


def test_rotary_refuses(lib):
    # B = 0 is a no-op; what is refused is refused before that
    assert _rotary(lib) == cp.CP_OK
    assert _rotary(lib, B=1, T=0) == cp.CP_OK
    assert _rotary(lib, rows(heads=0), B=1) == cp.CP_OK
    bad = [dict(dt=2), dict(n=0), dict(n=5), dict(B=-1), dict(T=-1), dict(D=0), dict(D=5000), dict(inverse=2),
           dict(rp=rope(rot=130)), dict(rp=rope(rot=7)), dict(rp=rope(rot=-2)), dict(rp=rope(layout=2)),
           dict(rp=rope(scale=float("inf"))), dict(rp=rope(inv_freq=None)), dict(rp=rope(inv_freq=FAKE + 4)),
           dict(r=rows(heads=-1)), dict(r=rows(in_=None)), dict(r=rows(out=None)), dict(r=rows(in_=FAKE + 1)),
           dict(r=rows(out=FAKE + 2), dt=0), dict(B=1, pos=0), dict(B=1, pos=FAKE + 4)]
    for b in bad:
        assert _rotary(lib, **b) == cp.CP_EINVAL, b
    assert lib.coverprune_rotary(None, 1, 1, 0, 1, 128, P(FAKE), 0, C.byref(rope()), 0, None) == cp.CP_EINVAL
    assert lib.coverprune_rotary(C.byref(rows()), 1, 1, 0, 1, 128, P(FAKE), 0, None, 0, None) == cp.CP_EINVAL


BAD_CACHES = [(dict(struct_size=8), cp.CP_EINVAL), (dict(dtype=3), cp.CP_EINVAL), (dict(heads=0), cp.CP_EINVAL),
              (dict(page_size=0), cp.CP_EINVAL), (dict(pages=-1), cp.CP_EINVAL), (dict(table_width=-1), cp.CP_EINVAL),
              (dict(D=260), cp.CP_EUNSUPPORTED), (dict(D=12), cp.CP_EUNSUPPORTED), (dict(D=0), cp.CP_EINVAL),
              (dict(slot_stride=4), cp.CP_EINVAL), (dict(head_stride=12), cp.CP_EINVAL),
              (dict(page_stride=1), cp.CP_EINVAL), (dict(page_size=1 << 30, table_width=8), cp.CP_EUNSUPPORTED)]
BAD_MEMORY = [(dict(k=None), cp.CP_EINVAL), (dict(v=FAKE + 8), cp.CP_EINVAL), (dict(table=None), cp.CP_EINVAL),
              (dict(table=FAKE + 2), cp.CP_EINVAL), (dict(k_scale=FAKE + 1), cp.CP_EINVAL)]


def _append(lib, c=None, k=FAKE, v=FAKE, dt=1, T=3, starts=FAKE, lens=FAKE, B=2, pos=FAKE, rp=None, q=None, new=None,
            status=None):
    st = TWO(512, 128)
    return lib.coverprune_cache_append(C.byref(c or cache()), P(k), st, P(v), st, dt, T, P(starts), P(lens), B, P(pos),
                                       C.byref(rp or rope()), None if q is None else C.byref(q), P(new), P(status), None)


def test_append_refuses(lib):
    assert _append(lib, B=0) == cp.CP_OK          # every row is padding
    assert _append(lib, T=0) == cp.CP_OK
    for c, want in BAD_CACHES + BAD_MEMORY:
        assert _append(lib, cache(**c), T=0) == want, c
    assert _append(lib, cache(dtype=cp.CP_F32)) == cp.CP_EUNSUPPORTED       # bf16 rows into a float32 cache
    assert _append(lib, dt=0) == cp.CP_EUNSUPPORTED
    for b in (dict(dt=2), dict(T=-1), dict(B=-1), dict(starts=0), dict(lens=0), dict(lens=FAKE + 2), dict(pos=FAKE + 4),
              dict(new=FAKE), dict(new=FAKE + 2), dict(status=FAKE + 1), dict(k=0), dict(v=FAKE + 1), dict(rp=rope(rot=256)),
              dict(q=rows(in_=None))):
        assert _append(lib, **b) == cp.CP_EINVAL, b


def _decode(lib, c=None, q=FAKE, dt=1, B=2, Hq=28, lens=FAKE, scale=0.1, window=0, out=FAKE, lse=None, ws=FAKE,
            ws_bytes=1 << 40, status=None):
    st = TWO(3584, 128)
    return lib.coverprune_decode_attention(P(q), st, dt, B, Hq, C.byref(c or cache()), P(lens), None, 0, scale, window,
                                           P(out), st, P(lse), P(ws), ws_bytes, P(status), None)


def test_decode_refuses(lib):
    assert _decode(lib, B=0) == cp.CP_OK
    assert _decode(lib, Hq=0) == cp.CP_OK
    for c, want in BAD_CACHES + BAD_MEMORY:
        assert _decode(lib, cache(**c), B=0) == want, c
    assert _decode(lib, cache(dtype=cp.CP_F32)) == cp.CP_EUNSUPPORTED
    assert _decode(lib, cache(dtype=cp.CP_E4M3), dt=0) == cp.CP_EUNSUPPORTED
    assert _decode(lib, B=1 << 23) == cp.CP_EUNSUPPORTED
    for b in (dict(dt=2), dict(B=-1), dict(Hq=27), dict(Hq=-4), dict(scale=float("nan")), dict(window=-1), dict(q=0),
              dict(q=FAKE + 1), dict(out=0), dict(out=FAKE + 1), dict(lens=0), dict(lse=FAKE + 2), dict(status=FAKE + 1)):
        assert _decode(lib, **b) == cp.CP_EINVAL, b
    # pages spread over more than 2^32 of the largest unit their strides share (16 bytes)
    assert _decode(lib, cache(pages=0x7FFFFFFF, page_stride=16 * 512 + 8)) == cp.CP_EUNSUPPORTED
    assert _decode(lib, cache(slot_stride=-512), B=0) == cp.CP_EINVAL
    for b in (dict(ws=0), dict(ws=FAKE + 128), dict(ws_bytes=16)):
        assert _decode(lib, **b) == cp.CP_EWORKSPACE, b


def test_decode_workspace(lib):
    def size(B, Hq, **kw):
        n = C.c_size_t()
        st = lib.coverprune_decode_workspace_size(B, Hq, C.byref(cache(k=None, v=None, table=None, **kw)), C.byref(n))
        assert st == cp.CP_OK
        return n.value

    assert size(1, 4) <= size(1, 28) <= size(64, 28) <= size(300, 64)
    for c, want in BAD_CACHES:
        n = C.c_size_t()
        assert lib.coverprune_decode_workspace_size(1, 4, C.byref(cache(**c)), C.byref(n)) == want
    assert lib.coverprune_decode_workspace_size(1, 4, C.byref(cache()), None) == cp.CP_EINVAL


def test_python_refuses_cpu_tensors():
    x, pos, f = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int64), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError):
        cp.coverprune_rotary(x, pos, f)
    pool, table, lens = torch.zeros(4, 16, 2, 64), torch.zeros(3, 1, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        cp.coverprune_cache_append(x, x, pool, pool, table, lens)
    with pytest.raises(ValueError):
        cp.coverprune_decode_attention(x, pool, pool, table, lens)
