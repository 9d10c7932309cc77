"""Pages that another request holds are read only: page tables refuse steps that would write into them."""
import pytest
import torch

import paper_2510_11958_amd as pkg
from test_gpu_paged import DEV, Maps, ints

pytestmark = pytest.mark.gpu


def state(t):
    return [x.clone() for x in (t.block_table, t.held, t.free_pages, t.n_free)]


def refused(t, m, start, rows, shared, who):
    was = state(t)
    m.pos.fill_(-6)
    m.slots.fill_(-7)
    t.build(ints(start), ints(rows), *m.all(), shared=ints(shared))
    assert m.status.tolist() == [pkg.DMTD_EINVAL, who] and not m.cu.any()
    assert (m.pos == -6).all() and (m.slots == -7).all()
    for a, b in zip(was, state(t)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("n_req, room", [(4, 64), (80, 512), (300, 1024), (300, 4096)])
def test_rows_inside_shared_pages_are_refused(n_req, room, page):
    """In each of the layouts that the tables are built in: requests 1, 3, .. stand behind two pages of request 0's."""
    t, m = pkg.PageTables.empty(4 * n_req + 4, page, n_req, 6, DEV), Maps(n_req, room)
    zero = [0] * n_req
    t.build(ints([0] * n_req), ints([2 * page if page == 16 else 20] + zero[1:]), *m.all())
    if page > 16:
        t.build(ints([2 * page - 3] + zero[1:]), ints([3] + zero[1:]), *m.all())
    assert t.held[0].item() == 2
    behind = list(range(1, n_req, 2))
    for i in behind:
        t.block_table[i, :2] = t.block_table[0, :2]
        t.held[i] = 2
    shared = [2 if i in behind else 0 for i in range(n_req)]
    start = [2 * page] + [2 * page if i in behind else 0 for i in range(1, n_req)]
    rows = [0] + [1] * (n_req - 1)
    last = behind[-1]

    def but(a, **kw):
        return [kw.get("_%d" % i, x) for i, x in enumerate(a)]

    for bad in (2 * page - 1, 0, page, 1):                                          # the last shared place, the first one, those between
        refused(t, m, but(start, **{"_%d" % last: bad}), rows, shared, last)
    refused(t, m, but(start, **{"_%d" % last: 0}), but(rows, **{"_%d" % last: 2 * page + 1}) if 2 * page + 1 + n_req < room else rows, shared, last)      # rows that reach beyond the pages too
    refused(t, m, but(start, _1=2 * page - 1, **{"_%d" % last: 0}), rows, shared, 1)      # the first such request is named
    # without rows, lengths inside the shared pages are fine: a request that has ended, or has been stepped back
    t.build(ints(but(start, _1=2 * page - 1, **{"_%d" % last: 0})), ints(but(rows, _1=0, **{"_%d" % last: 0})), *m.all(), shared=ints(shared))
    assert m.status.tolist() == [0, 0] and m.cu[-1].item() == n_req - 1 - len({1, last})
    assert (t.held[behind] == torch.tensor([2 if i in (1, last) else 3 for i in behind], device=DEV)).all()
    # and the first place behind them is the first that may be written
    t.build(ints(start), ints(rows), *m.all(), shared=ints(shared))
    assert m.status.tolist() == [0, 0]
    front = set(t.block_table[0, :2].tolist())
    assert front.isdisjoint((m.slots[:n_req - 1] // page).tolist()) and (t.held[behind] == 3).all()


def test_pages_of_ones_own_may_be_written():
    """The holder's step back and on again, and a request that shares fewer pages than it holds."""
    t, m = pkg.PageTables.empty(8, 16, 2, 4, DEV), Maps(2, 64)
    t.build(ints([0, 0]), ints([40, 0]), *m.all())
    t.block_table[1, :1] = t.block_table[0, :1]
    t.held[1] = 1
    t.build(ints([20, 16]), ints([5, 20]), *m.all(), shared=ints([0, 1]))
    assert m.status.tolist() == [0, 0]
    t.build(ints([10, 17]), ints([2, 3]), *m.all(), shared=ints([0, 1]))
    assert m.status.tolist() == [0, 0] and m.pos[:5].tolist() == [10, 11, 17, 18, 19]
    refused(t, m, [10, 15], [2, 3], [0, 1], 1)
