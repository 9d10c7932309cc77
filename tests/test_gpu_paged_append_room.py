"""An append's row_pos and slots have as many entries as dmtd_page_tables was given room for, which may be fewer than the cache handle's rows: none behind the step's last row is read."""
import ctypes as C

import pytest
import torch

import paged_util as pu
import paper_2510_11958_amd as pkg
from test_gpu_paged import BF, DEV, F32, H4, H8, Setup, ints
from test_gpu_paged8 import E8, Setup8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32, E8])
@pytest.mark.parametrize("heads, start, rows", [(H8, [5, 40], [1, 2]), (H4, [0], [1]), (H8, [0, 16, 3], [70, 0, 1])])
def test_maps_of_fewer_rows_than_the_handle(heads, start, rows, dtype):
    pools = []
    for maps_room in ("the step's", "the handle's"):
        s = (Setup8(heads, 16, start, rows, seed=4, room=4096) if dtype is E8 else Setup(heads, dtype, 16, start, rows, seed=4, room=4096))
        c = s.cache()
        n = s.total if maps_room == "the step's" else s.room
        pad = n - s.total
        pos, slots = ints(s.pos + [-1] * pad), ints(s.slots + [-1] * pad, torch.int64)
        qkv = s.qkv[:n].contiguous().to(DEV)
        gain, rope = s.dev(s.gain), s.dev(s.rope)
        lib = pkg.load_library()
        rc = lib.dmtd_paged_append(C.byref(c._c), qkv.data_ptr(), qkv.shape[1], ints(s.cu).data_ptr(), pos.data_ptr(), slots.data_ptr(), gain.data_ptr(), pu.EPS, rope.data_ptr(), rope.shape[0],
                                   torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert rc == pkg.DMTD_OK
        pools.append([t.view(torch.uint8).cpu() for t in ((s.kd, s.vd, s.ksd, s.vsd) if dtype is E8 else (s.kd, s.vd))])
        was = [t.contiguous().view(torch.uint8) for t in ((s.kb, s.vb) if dtype is E8 else (s.k, s.v))]
        assert not any(torch.equal(a, b) for a, b in zip(pools[-1], was))      # (the scales' powers may be what they were)
    for a, b in zip(*pools):
        assert torch.equal(a, b)
