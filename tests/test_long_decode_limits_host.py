"""Memory that the calls of a long decode must not share, and sizes at their limits: refused before anything is launched (fake
pointers, never dereferenced)."""
import ctypes as C

import pytest

import paper_2608_13226_gb300 as cp
from test_serve_host import P, TWO, cache, lib  # noqa: F401

FAR = 1 << 32  # addresses that do not overlap
Q, OUT, LENS, LSE, WEIGHT, KEEP, WS = (i * FAR for i in range(1, 8))
B, HQ, D, KEYS = 3, 28, 128, 128  # a cache of 8 pages of 16 a row


def _weigh(lib, q=Q, q_st=(HQ * D, D), out=OUT, out_st=(HQ * D, D), lse=LSE, lens=LENS, keep=KEEP, keep_stride=KEYS, weight=WEIGHT, stride=KEYS, ws=WS):
    n, c = C.c_size_t(), cache()
    assert lib.coverprune_decode_weigh_workspace_size(B, HQ, C.byref(c), C.byref(n)) == cp.CP_OK
    return lib.coverprune_decode_attention_weigh(P(q), TWO(*q_st), cp.CP_BF16, B, HQ, C.byref(c), P(lens), P(keep), keep_stride, 0.1, 0, P(out),
                                                 TWO(*out_st), P(lse), P(weight), stride, P(ws), n.value, None, None), n.value


ROW = 2 * HQ * D       # bytes of a sequence's queries or outputs, bfloat16
W = 4 * KEYS           # of its weights


@pytest.mark.parametrize("kw", [
    dict(weight=Q), dict(weight=Q - W), dict(weight=Q + 3 * ROW - 4), dict(weight=OUT), dict(weight=OUT + 3 * ROW - 4), dict(weight=OUT - 3 * W + 4),
    dict(weight=OUT + ROW // 2, stride=HQ * D // 2),  # rows take turns at the outputs' distance, but in their place
    dict(weight=OUT + ROW + 4 - W, out_st=(HQ * D + 2 * KEYS, D), stride=HQ * D // 2 + KEYS),
    dict(weight=OUT - 4 * ROW, out=OUT - 2 * ROW, out_st=(-HQ * D, D), stride=1 << 20), dict(out=OUT, out_st=(0, -D), weight=OUT - ROW + 2 * D),
    dict(weight=LSE + 4 * B * HQ - 4), dict(weight=LENS), dict(weight=LENS + 8), dict(weight=KEEP + 2 * KEYS), dict(weight=KEEP, keep_stride=0),
    dict(weight=WS), dict(weight=WS - 3 * W + 4)])
def test_weights_in_place_of_others(lib, kw):
    st, _ = _weigh(lib, **kw)
    assert st == cp.CP_EINVAL, kw


def test_weights_in_the_workspace_end(lib):
    _, n = _weigh(lib, weight=Q)
    assert _weigh(lib, weight=WS + n - 4)[0] == cp.CP_EINVAL


def test_most_keys_that_evictions_leave(lib):
    """B * left < 2^35, as the header says: the largest is looked at further (and lacks its lengths), the next one is too much."""
    def evict(B, left):
        return lib.coverprune_cache_evict(C.byref(cache()), None, B, P(WEIGHT), KEYS, left, 0, 0, None, None, 0, 0, P(OUT), None, None)

    assert 279527 * 122921 == 2 ** 35 - 1
    assert evict(279527, 122921) == cp.CP_EINVAL
    assert evict(1 << 15, 1 << 20) == cp.CP_EUNSUPPORTED and evict(1 << 24, 1 << 30) == cp.CP_EUNSUPPORTED
