"""Calls of the paged cache's operators that the device or the handles refuse, and the calls behind them."""
import pytest
import torch

import paper_2510_11958_amd as pkg
from test_gpu_paged import BF, DEV, H8, Setup, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_req", [62, 130])
def test_rows_that_descend(n_req):
    """Requests that share rows bring more groups than a launch has blocks for (the 20 in front of the long one 80, it four in 22 key ranges each; 144 blocks): no row comes out, and
    the handle's next call, whose groups count their ranges in the same places, is right."""
    at = 40
    s = Setup(H8, BF, 16, [0] * at + [4080] + [0] * (n_req - at - 1), [0] * at + [16] + [0] * (n_req - at - 1), seed=41, room=16)
    c, cu = s.cache(), ints([0, 16] * (n_req // 2) + [0])
    for _ in range(2):
        out = torch.full((s.room, s.nq, s.hd), 77.0, dtype=BF, device=DEV)
        c.attention(s.qkv.to(DEV), ints(s.start), cu, out, q_norm=s.dev(s.gain), rope=s.dev(s.rope))
        assert (out == 77.0).all()
        s.check(s.attend(c))
    # (one request starts below 0: the same)
    out = torch.full((s.room, s.nq, s.hd), 77.0, dtype=BF, device=DEV)
    c.attention(s.qkv.to(DEV), ints(s.start), ints([-1] + s.cu[1:]), out, q_norm=s.dev(s.gain), rope=s.dev(s.rope))
    assert (out == 77.0).all()
    s.check(s.attend(c))
