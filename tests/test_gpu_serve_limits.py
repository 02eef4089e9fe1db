"""The decoding model's operators at the edges of what they take: arguments that
are refused, values at the ends of a type, and the bounds that the header states."""
import pytest
import torch

import paper_2608_13226_gb300 as cp

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
BF16, F32 = torch.bfloat16, torch.float32


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
