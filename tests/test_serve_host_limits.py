"""Arguments of the decoding model's entry points that the host refuses, beside those of
test_serve_host.py (fake pointers, never dereferenced)."""
import pytest

import paper_2608_13226_gb300 as cp
from test_serve_host import FAKE, _append


@pytest.fixture(scope="module")
def lib():
    from paper_2608_13226_gb300 import build
    build.build()
    return cp.load()


@pytest.mark.parametrize("B", [1, 2, 100])
def test_new_lengths_that_overlap_are_refused(lib, B):
    """Not only at the same address: any shared element would be read by some blocks while
    others write it."""
    lens, starts = FAKE, FAKE + (1 << 20)
    for at in (lens, lens + 4 * (B - 1), lens - 4 * (B - 1), starts, starts + 4 * B, starts - 4 * (B - 1)):
        assert _append(lib, lens=lens, starts=starts, new=at, B=B) == cp.CP_EINVAL, at - FAKE
