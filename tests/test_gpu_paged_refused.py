"""Calls of the paged cache's operators that the device or the handles refuse, and the calls behind them."""
import pytest
import torch

import paged_util as pu
import paper_2510_11958_amd as pkg
from test_gpu_paged import BF, DEV, H8, Setup, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_req", [62, 130])
def test_rows_that_descend(n_req):
    """Requests that share rows bring more groups than a launch has blocks for (the 20 in front of the long one 80, it four in 22 key ranges each; 144 blocks, so that its third
    group misses two ranges): no row comes out, and the handle's next calls, whose groups count up to 32 and 16 ranges in the same place, are right."""
    at = 40
    s = Setup(H8, BF, 16, [0] * at + [4080] + [0] * (n_req - at - 1), [0] * at + [16] + [0] * (n_req - at - 1), seed=41, room=16)
    shorter = [2000 if i == at else 0 for i in range(n_req)]
    ref, tol = pu.attention(s.qkv, s.nq, s.k, s.v, s.table, 16, shorter, s.rows, s.gain, s.rope, True)
    c = s.cache()

    def attend(start, cu):
        out = torch.full((s.room, s.nq, s.hd), 77.0, dtype=BF, device=DEV)
        c.attention(s.qkv.to(DEV), ints(start), ints(cu), out, q_norm=s.dev(s.gain), rope=s.dev(s.rope))
        return out.cpu()

    for cu in ([0, 16] * (n_req // 2) + [0], [-1] + s.cu[1:]):
        out = attend(s.start, cu)
        assert ((attend(shorter, s.cu).double() - ref).abs() <= tol).all()
        s.check(attend(s.start, s.cu))
        assert (out == 77.0).all()


def test_pages_that_overlap():
    """One page expanded to many has a stride of 0, which the C call takes for pages that follow each other; others lie closer than a page is long."""
    table = ints([[0, 1]])
    for dtype in (BF, torch.float32):
        page = torch.zeros(1, 2, 16, 64, dtype=dtype, device=DEV)
        close = torch.zeros(9 * 1024 + 2048, dtype=dtype, device=DEV).as_strided((10, 2, 16, 64), (1024, 1024, 64, 1))
        for k in (page.expand(10, 2, 16, 64), close):
            with pytest.raises(ValueError):
                pkg.PagedCache(k, k, table, 4, 8)
        pkg.PagedCache(page, page, table, 4, 8)


def test_an_empty_rotary_table():
    """Not "no rotation", although its address is null."""
    s = Setup(H8, BF, 16, [20], [3], seed=42)
    c, none = s.cache(), torch.zeros(0, s.hd // 2, 2, device=DEV)
    qkv, cu, pad = s.qkv.to(DEV), ints(s.cu), s.room - s.total
    with pytest.raises(ValueError):
        c.attention(qkv, ints(s.start), cu, q_norm=s.dev(s.gain), rope=none)
    with pytest.raises(ValueError):
        c.append(qkv, cu, ints(s.pos + [-1] * pad), ints(s.slots + [-1] * pad, torch.int64), k_norm=s.dev(s.gain), rope=none)
    torch.cuda.synchronize()
    assert torch.equal(s.kd.cpu().view(torch.int16), s.k.view(torch.int16))
