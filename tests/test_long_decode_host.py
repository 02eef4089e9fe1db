"""What the calls on 4-bit caches, the weights of keys, reading and eviction refuse before anything is launched (fake
pointers, never dereferenced), and the sizes of their workspaces."""
import ctypes as C

import pytest
import torch

import paper_2608_13226_gb300 as cp
from paper_2608_13226_gb300 import binding
from test_serve_host import BAD_CACHES, BAD_MEMORY, FAKE, P, TWO, _append, _decode, cache, lib  # noqa: F401


def fours(**kw):
    """A cache of 4 bits: 10 pages of 16 rows of 4 heads of 128."""
    return cache(**{**dict(dtype=cp.CP_I4, k_block=FAKE, v_block=FAKE, block_page_stride=16 * 32, block_slot_stride=32, block_head_stride=8), **kw})


BAD_FOURS = [(dict(D=48), cp.CP_EUNSUPPORTED), (dict(D=16), cp.CP_EUNSUPPORTED), (dict(slot_stride=16), cp.CP_EINVAL), (dict(head_stride=8), cp.CP_EINVAL),
             (dict(page_stride=33), cp.CP_EINVAL), (dict(block_page_stride=-4), cp.CP_EINVAL), (dict(block_slot_stride=2), cp.CP_EINVAL),
             (dict(block_head_stride=1), cp.CP_EINVAL), (dict(struct_size=binding._Cache.k_block.offset), cp.CP_EINVAL)]
BAD_BLOCKS = [(dict(k_block=None), cp.CP_EINVAL), (dict(v_block=None), cp.CP_EINVAL), (dict(k_block=FAKE + 2), cp.CP_EINVAL)]


def test_struct_without_blocks_is_taken(lib):
    """A caller compiled before there were 4-bit caches passes a shorter struct."""
    short = dict(struct_size=binding._Cache.k_block.offset)
    assert _append(lib, cache(**short), T=0) == cp.CP_OK
    assert _decode(lib, cache(**short), B=0) == cp.CP_OK
    assert _decode(lib, cache(struct_size=short["struct_size"] - 8), B=0) == cp.CP_EINVAL


def test_fours_are_refused(lib):
    assert _append(lib, fours(), T=0) == cp.CP_OK and _append(lib, fours(), T=0, dt=0) == cp.CP_OK
    assert _decode(lib, fours(), B=0) == cp.CP_OK
    for c, want in BAD_FOURS + BAD_BLOCKS:
        assert _append(lib, fours(**c), T=0) == want, c
        assert _decode(lib, fours(**c), B=0) == want, c
    assert _decode(lib, fours(), dt=0) == cp.CP_EUNSUPPORTED
    assert _decode(lib, fours(pages=0x7FFFFFFF, block_page_stride=(1 << 20) + 4)) == cp.CP_EUNSUPPORTED


def _weigh(lib, c=None, q=FAKE, dt=1, B=2, Hq=28, lens=FAKE, scale=0.1, window=0, out=FAKE, lse=None, weight=FAKE, stride=128, ws=FAKE,
           ws_bytes=1 << 40, status=None):
    st = TWO(3584, 128)
    return lib.coverprune_decode_attention_weigh(P(q), st, dt, B, Hq, C.byref(c or cache()), P(lens), None, 0, scale, window, P(out), st,
                                                 P(lse), P(weight), stride, P(ws), ws_bytes, P(status), None)


def test_weigh_refuses(lib):
    assert _weigh(lib, B=0) == cp.CP_OK and _weigh(lib, Hq=0) == cp.CP_OK
    for c, want in BAD_CACHES + BAD_MEMORY:
        assert _weigh(lib, cache(**c), B=0) == want, c
    for c, want in BAD_FOURS + BAD_BLOCKS:
        assert _weigh(lib, fours(**c), B=0) == want, c
    for b in (dict(dt=2), dict(B=-1), dict(Hq=27), dict(scale=float("nan")), dict(window=-1), dict(q=0), dict(out=0), dict(lens=0), dict(weight=0),
              dict(weight=FAKE + 2), dict(stride=-1), dict(stride=127), dict(status=FAKE + 1), dict(lse=FAKE + 2)):
        assert _weigh(lib, **b) == cp.CP_EINVAL, b
    assert _weigh(lib, cache(dtype=cp.CP_F32)) == cp.CP_EUNSUPPORTED
    for b in (dict(ws=0), dict(ws=FAKE + 128), dict(ws_bytes=16)):
        assert _weigh(lib, **b) == cp.CP_EWORKSPACE, b
    n, m = C.c_size_t(), C.c_size_t()
    for c in (cache(), fours()):
        assert lib.coverprune_decode_weigh_workspace_size(2, 28, C.byref(c), C.byref(n)) == cp.CP_OK
        assert lib.coverprune_decode_workspace_size(2, 28, C.byref(c), C.byref(m)) == cp.CP_OK
        assert n.value >= m.value + 4 * 2 * 28 * (1 + 128)  # 8 pages of 16 a row
        assert _weigh(lib, c, ws_bytes=n.value - 1) == cp.CP_EWORKSPACE
        assert _decode(lib, c, ws_bytes=m.value - 1) == cp.CP_EWORKSPACE
    assert lib.coverprune_decode_weigh_workspace_size(1, 4, C.byref(cache()), None) == cp.CP_EINVAL
    # a size that 64 bits do not hold is refused, not cut
    vast = cache(heads=1, table_width=1 << 26)
    assert lib.coverprune_decode_weigh_workspace_size(1 << 24, 1 << 16, C.byref(vast), C.byref(n)) == cp.CP_EUNSUPPORTED
    assert _weigh(lib, vast, B=1 << 24, Hq=1 << 16, stride=1 << 30) == cp.CP_EUNSUPPORTED
    for c, want in BAD_CACHES:
        assert lib.coverprune_decode_weigh_workspace_size(1, 4, C.byref(cache(**c)), C.byref(n)) == want


def _read(lib, c=None, T=3, starts=FAKE, lens=FAKE, B=2, k=FAKE, v=FAKE, dt=1, status=None):
    st = TWO(512, 128)
    return lib.coverprune_cache_read(C.byref(c or cache()), T, P(starts), P(lens), B, P(k), st, P(v), st, dt, P(status), None)


def test_read_refuses(lib):
    assert _read(lib, B=0) == cp.CP_OK and _read(lib, T=0) == cp.CP_OK and _read(lib, fours(), T=0, dt=0) == cp.CP_OK
    for c, want in BAD_CACHES + BAD_MEMORY:
        assert _read(lib, cache(**c), T=0) == want, c
    for c, want in BAD_FOURS + BAD_BLOCKS:
        assert _read(lib, fours(**c), T=0) == want, c
    assert _read(lib, dt=0) == cp.CP_EUNSUPPORTED and _read(lib, cache(dtype=cp.CP_F32)) == cp.CP_EUNSUPPORTED
    for b in (dict(dt=2), dict(T=-1), dict(B=-1), dict(starts=0), dict(lens=0), dict(lens=FAKE + 2), dict(starts=FAKE + 1), dict(k=0), dict(v=FAKE + 1),
              dict(status=FAKE + 2), dict(B=1 << 25)):
        assert _read(lib, **b) == cp.CP_EINVAL, b


FAR = 1 << 30  # addresses that do not overlap


def _evict(lib, c=None, lens=FAKE, B=2, weight=FAKE + FAR, stride=128, left=10, first=1, recent=2, new_lens=FAKE + 2 * FAR, new_weight=FAKE + 3 * FAR,
           new_stride=128, width=128, kept=FAKE + 4 * FAR, status=None):
    return lib.coverprune_cache_evict(C.byref(c or cache()), P(lens), B, P(weight), stride, left, first, recent, P(new_lens), P(new_weight), new_stride,
                                      width, P(kept), P(status), None)


def test_evict_refuses(lib):
    assert _evict(lib, B=0) == cp.CP_OK
    for c, want in BAD_CACHES + BAD_MEMORY:
        assert _evict(lib, cache(**c), B=0) == want, c
    for c, want in BAD_FOURS + BAD_BLOCKS:
        assert _evict(lib, fours(**c), B=0) == want, c
    for b in (dict(B=-1), dict(left=-1), dict(first=-1), dict(recent=-1), dict(first=11), dict(first=5, recent=6), dict(first=1 << 62, recent=1 << 62),
              dict(lens=0), dict(lens=FAKE + 1), dict(weight=0), dict(weight=FAKE + FAR + 2), dict(stride=-1), dict(new_stride=-1), dict(new_stride=127), dict(stride=1 << 60),
              dict(new_stride=1 << 60),
              dict(width=-1), dict(kept=0), dict(kept=FAKE + 4 * FAR + 1), dict(new_lens=FAKE), dict(new_lens=FAKE + FAR + 4), dict(new_weight=FAKE + FAR + 512),
              dict(new_weight=FAKE + FAR - 1020), dict(kept=FAKE + FAR + 1020), dict(kept=FAKE + 3 * FAR + 4), dict(kept=FAKE + 2 * FAR + 4), dict(kept=FAKE),
              dict(status=FAKE + 1)):
        assert _evict(lib, **b) == cp.CP_EINVAL, b
    assert _evict(lib, B=1 << 20, left=1 << 20, weight=1 << 50, kept=1 << 52, new_lens=None, new_weight=None) == cp.CP_EUNSUPPORTED


def test_python_refuses_cpu_tensors():
    x, table, lens = torch.zeros(3, 2, 64), torch.zeros(3, 1, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    held, blocks = torch.zeros(4, 16, 2, 32, dtype=torch.uint8), torch.zeros(4, 16, 2, 4).to(torch.float8_e4m3fn)
    kw = dict(k_block=blocks, v_block=blocks)
    for f in (lambda: cp.coverprune_cache_append(x, x, held, held, table, lens, **kw),
              lambda: cp.coverprune_cache_read(held, held, table, lens, **kw),
              lambda: cp.coverprune_decode_attention(x, held, held, table, lens, **kw),
              lambda: cp.coverprune_cache_evict(held, held, table, lens, torch.zeros(3, 16), 4, **kw)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        cp.coverprune_cache_read(held, held, table, lens, dtype=torch.float16, **kw)


def test_keys_and_values_in_one_place(lib):
    """Writes to both would meet; before anything else is looked at that needs a device."""
    far = FAKE + 5 * FAR
    for c in (fours(k=far, v=far), fours(v=FAKE + FAR, k_block=far, v_block=far)):
        assert _append(lib, c, T=3) == cp.CP_EINVAL
        assert _evict(lib, c) == cp.CP_EINVAL
    assert _evict(lib, cache(k=far, v=far)) == cp.CP_EINVAL
    assert _read(lib, k=far, v=far) == cp.CP_EINVAL
