"""The paged cache's operators where steps are large: the layouts and branches that small cases do not reach, against the plain 64-bit forms.  What each case reaches is worked out
here by the launches' own rules (a test without a GPU holds it)."""
import numpy as np
import pytest
import torch

import paged_util as pu
import paper_2510_11958_amd as pkg
from test_gpu_paged import BF, DEV, F32, Maps, Setup, check_step, ints

RESIDENT, SLOTS, FEW, MIN_KEYS, TILE = 512, 256, 64, 256, 64      # of the kernel for many rows of a request (attention_paged.hpp)


def ceil(a, b):
    return -(-a // b)


def layout(heads, start, rows, room):
    """How the kernel for many rows lays a step out: (keys of a range, most ranges of a group, items per KV head, items of the first round of the CUs, vectors a thread of the merge takes)."""
    nq, nkv, hd = heads
    gq = nq // nkv
    rpb, shift = 128 // gq, (SLOTS // nkv).bit_length() - 1
    mine = [(ceil(r, rpb), s + r) for s, r in zip(start, rows) if r * gq > FEW]
    keys = max(MIN_KEYS, ceil(ceil(sum(g * k for g, k in mine), 1 << shift), TILE) * TILE)
    items = sum(g * ceil(k, keys) for g, k in mine)
    down = min(items, ceil(RESIDENT // 2, nkv)) if items * nkv <= RESIDENT else items
    groups = min(len(start), room // (FEW // gq + 1)) + room // rpb
    blocks = min(hd // 8, max(hd // 32, 1024 // (nkv * min(groups, 1 << shift))))
    return keys, max(ceil(k, keys) for _, k in mine), items, down, hd // 8 // blocks


CASES = {
    # heads, page, start, rows, room, what the layout is
    "ranges from the sum of the keys": ((16, 8, 128), 64, [3000, 100, 5000], [140, 1, 90], 240, (640, 8, 31, 31, 1)),
    "a second round, ranges": ((8, 2, 64), 32, [8000], [130], 136, (320, 26, 130, 128, 1)),
    "a second round, one range": ((128, 128, 64), 16, [0], [300], 304, (512, 1, 3, 2, 2)),
    "more blocks than are resident": ((128, 128, 64), 16, [0, 5], [600, 130], 736, (1664, 1, 7, 7, 2)),
    "more blocks than are resident, ranges": ((128, 128, 64), 16, [3000, 0], [100, 512], 616, (2624, 2, 6, 6, 2)),
    "a merge of two vectors a thread": ((8, 2, 64), 16, [8000, 3], [130, 2], 4096, (320, 26, 130, 128, 2)),
    "a merge of four vectors a thread": ((8, 2, 128), 256, [700, 7000], [100, 77], 4096, (256, 28, 100, 100, 4)),
    "a long chunk": ((8, 2, 128), 16, [1000], [1500], 1504, (960, 3, 141, 128, 1)),
}


@pytest.mark.parametrize("name", list(CASES))
def test_what_the_cases_reach(name):
    heads, page, start, rows, room, want = CASES[name]
    assert layout(heads, start, rows, room) == want


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_many_rows(name):
    heads, page, start, rows, room, _ = CASES[name]
    s = Setup(heads, BF, page, start, rows, seed=51, room=room)
    got = s.attend()
    s.check(got)
    assert torch.equal(s.attend(max_new=max(rows)), got)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, rows", [(BF, 130), (BF, 9), (F32, 9)])
def test_values_and_pages_in_several_ranges(dtype, rows):
    """A page missing from a range, one of the chunk's own values not finite: rows that see that one are NaN or infinite in its dim, the others right."""
    def setup():
        s = Setup((8, 2, 64), dtype, 32, [8000], [rows], seed=52)
        s.table[0][100] = -1
        s.table[0][203] = s.n_pages
        return s

    s = setup()
    s.check()
    mid, last = rows // 2, 8000 + rows // 2
    s.v[s.table[0][last // 32], :, last % 32, 5] = float("inf")
    got, (ref, tol) = s.attend(), setup().reference()
    assert ((got[:mid].double() - ref[:mid]).abs() <= tol[:mid]).all()
    assert not torch.isfinite(got[mid:, :, 5]).any()


@pytest.mark.gpu
def test_tables_of_many_pages():
    """Steps of the three launches that move more than 2 x 2 x 16384 pages, which the blocks take two a thread and round: taken, given back while others take as many, given back, and mixed."""
    n, page, most = 60, 16, 1500
    tables, model = pkg.PageTables.empty(n * most, page, 2 * n, most, DEV), pu.Pool(n * most, page, 2 * n, most)
    rng = np.random.RandomState(6)
    lengths = (page * rng.randint(1200, most, n) - 3).tolist()
    none, ones, room = [0] * n, [1] * n, 2500
    assert sum(ceil(x + 1, page) for x in lengths) > 4 * 16384
    for start, rows in ((lengths + none, ones + none), (none + lengths, none + ones), (none + none, none + none), (lengths + none, ones + none),
                        ([x // 3 for x in lengths] + [x // 2 for x in lengths], ones + ones), (none + lengths, none + [3] * n)):
        check_step(tables, model, start, rows, room)
