"""The paged cache's operators against their plain 64-bit forms (paged_util), one by one and together."""
import numpy as np
import pytest
import torch

import paper_2510_11958_amd as pkg
import paged_util as pu

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(a, t=torch.int32):
    return torch.as_tensor(np.asarray(a, dtype=np.int64)).to(t).to(DEV)


class Maps:
    """A step's row maps with sentinels in them."""

    def __init__(self, n_req, room):
        self.cu, self.pos, self.slots, self.status = ints([-5] * (n_req + 1)), ints([-6] * room), ints([-7] * room, torch.int64), ints([9, 9])

    def all(self):
        return self.cu, self.pos, self.slots, self.status


# ------------------------------------------------------------------------------------------ bookkeeping

def check_step(tables, model, start, rows, room):
    m = Maps(len(start), room)
    tables.build(ints(start), ints(rows), *m.all())
    status, cu, pos, slots = model.step(start, rows, room)
    torch.cuda.synchronize()
    assert tuple(m.status.tolist()) == status
    assert m.cu.tolist() == cu
    assert m.pos.tolist() == pos + [-6] * (room - len(pos))
    assert m.slots.tolist() == slots + [-7] * (room - len(slots))
    assert tables.held.tolist() == model.held
    assert tables.block_table.tolist() == model.table
    assert tables.n_free.item() == len(model.free)
    assert tables.free_pages.tolist() == model.free + [-1] * (model.n_pages - len(model.free))


@pytest.mark.parametrize("n_req, page, max_pages, n_pages, room, most", [
    (1, 16, 4, 5, 16, 20), (3, 16, 6, 12, 64, 30), (64, 32, 5, 200, 64, 3), (65, 16, 9, 300, 2048, 60), (7, 256, 3, 15, 2049, 600), (300, 16, 40, 4000, 6000, 200),
    (1025, 16, 4, 2500, 5000, 25), (8192, 16, 2, 9000, 9000, 3), (8192, 32, 2, 8192, 2048, 1),
])
def test_page_tables_over_many_steps(n_req, page, max_pages, n_pages, room, most):
    rng = np.random.RandomState(n_req * 31 + page)
    tables, model = pkg.PageTables.empty(n_pages, page, n_req, max_pages, DEV), pu.Pool(n_pages, page, n_req, max_pages)
    start = np.zeros(n_req, int)
    for step in range(12):
        rows = rng.randint(0, most + 1, n_req) * (rng.rand(n_req) < rng.choice([0.1, 0.5, 1.0]))
        for i in np.nonzero(rng.rand(n_req) < 0.2)[0]:        # some end, some are rolled back by a few tokens
            start[i], rows[i] = (0, 0) if rng.rand() < 0.5 else (max(0, start[i] - rng.randint(0, 2 * page)), 0)
        over = start + rows > max_pages * page
        start[over], rows[over] = 0, 0
        while rows.sum() > room:
            rows[rng.randint(n_req)] = 0
            rows[np.argmax(rows)] //= 2
        check_step(tables, model, start.tolist(), rows.tolist(), room)
        if model.held == [-(-(s + r) // page) for s, r in zip(start, rows)]:
            start = start + rows


def test_refused_steps_change_nothing():
    tables, model = pkg.PageTables.empty(6, 16, 3, 4, DEV), pu.Pool(6, 16, 3, 4)
    check_step(tables, model, [0, 0, 0], [20, 0, 33], 64)                # 5 pages
    for start, rows in (([20, 0, 33], [1, 17, 15]),                       # lacks one page
                        ([20, 0, 33], [1, 65, -1]), ([20, 0, -1], [1, 0, 0]), ([20, 0, 33], [45, 0, 32]),      # lengths
                        ([20, 0, 33], [30, 30, 5])):                     # too many rows
        check_step(tables, model, start, rows, 64)
    check_step(tables, model, [20, 0, 33], [12, 16, 15], 64)             # takes the last page
    check_step(tables, model, [20, 0, 0], [13, 16, 0], 64)               # gives three back and takes one in the same step
    tables.held[1] = 5                                                   # what the pool does not hold together
    m = Maps(3, 64)
    tables.build(ints([1, 1, 1]), ints([1, 1, 1]), *m.all())
    assert m.status.tolist() == [-1, 1] and m.cu.tolist() == [0] * 4
    tables.held[1] = 1
    tables.n_free.fill_(7)
    tables.build(ints([1, 1, 1]), ints([1, 1, 1]), *m.all())
    assert m.status.tolist() == [-1, -1] and m.pos.tolist() == [-6] * 64


def test_giving_back_restores_the_stack():
    tables = pkg.PageTables.empty(50, 16, 4, 20, DEV)
    m = Maps(4, 512)
    tables.build(ints([0] * 4), ints([17, 40, 0, 5]), *m.all())
    before = [t.clone() for t in (tables.block_table, tables.held, tables.free_pages, tables.n_free)]
    tables.build(ints([17, 40, 0, 5]), ints([100, 1, 77, 200]), *m.all())
    assert tables.n_free.item() < before[3].item()
    tables.build(ints([17, 40, 0, 5]), ints([0] * 4), *m.all())
    for a, b in zip(before, (tables.block_table, tables.held, tables.free_pages, tables.n_free)):
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------ append and attention

class Setup:
    """Pages in random order behind random block tables; whatever no token lies in is NaN."""

    def __init__(self, heads, dtype, page, start, rows, seed=0, room=None, norm=True, rope=True, spread=1.0, extra_pages=3):
        self.nq, self.nkv, self.hd = heads
        self.dtype, self.page, self.start, self.rows = dtype, page, start, rows
        gen = torch.Generator().manual_seed(seed)
        rng = np.random.RandomState(seed)
        need = [-(-(s + r) // page) for s, r in zip(start, rows)]
        self.width, self.n_pages, self.total = max(need) + 1, sum(need) + extra_pages, sum(rows)
        self.room = room or max(self.total, 1) + 5
        order = rng.permutation(self.n_pages)
        self.table, at = [], 0
        for n in need:
            self.table.append(order[at:at + n].tolist() + [-1] * (self.width - n))
            at += n
        self.cu = np.concatenate([[0], np.cumsum(rows)]).tolist()
        self.pos = [p for s, r in zip(start, rows) for p in range(s, s + r)]
        self.slots = [self.table[i][p // page] * page + p % page for i, (s, r) in enumerate(zip(start, rows)) for p in range(s, s + r)]
        self.qkv = torch.randn(self.room, (self.nq + 2 * self.nkv) * self.hd, generator=gen) * spread
        self.qkv[self.total:] = float("nan")
        self.gain = (1 + 0.2 * torch.randn(self.hd, generator=gen)).to(dtype) if norm else None
        self.rope = pu.rope_table(self.width * page, self.hd) if rope else None
        shape = (self.n_pages, self.nkv, page, self.hd)
        self.k, self.v = torch.full(shape, float("nan"), dtype=dtype), torch.full(shape, float("nan"), dtype=dtype)
        for i, (s, r) in enumerate(zip(start, rows)):
            for j in range(-(-(s + r) // page)):
                n = min(page, s + r - j * page)
                self.k[self.table[i][j], :, :n] = torch.randn(self.nkv, n, self.hd, generator=gen).to(dtype)
                self.v[self.table[i][j], :, :n] = torch.randn(self.nkv, n, self.hd, generator=gen).to(dtype)

    def dev(self, t):
        return None if t is None else t.to(DEV)

    def cache(self, **kw):
        self.kd, self.vd = kw.pop("kv", None) or (self.k.to(DEV), self.v.to(DEV))
        return pkg.PagedCache(self.kd, self.vd, ints(self.table), self.nq, self.room)

    def reference(self):
        return pu.attention(self.qkv, self.nq, self.k, self.v, self.table, self.page, self.start, self.rows, self.gain, self.rope, self.dtype is torch.bfloat16)

    def attend(self, cache=None, max_new=0):
        out = torch.full((self.room, self.nq, self.hd), 77.0, dtype=self.dtype, device=DEV)
        (cache or self.cache()).attention(self.qkv.to(DEV), ints(self.start), ints(self.cu), out, q_norm=self.dev(self.gain), rope=self.dev(self.rope), eps=pu.EPS, max_new=max_new)
        torch.cuda.synchronize()
        assert (out[self.total:] == 77.0).all()
        return out[:self.total].cpu()

    def check(self, got=None):
        ref, tol = self.reference()
        got = self.attend() if got is None else got
        bad = ~((got.double() - ref).abs() <= tol)
        assert not bad.any(), (int(bad.sum()), (got.double() - ref).abs().max(), bad.nonzero()[:4].tolist())


H4, H8, H7, H1, H16, H6 = (4, 2, 64), (8, 2, 128), (7, 1, 64), (3, 3, 128), (16, 1, 128), (12, 2, 128)
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("heads, dtype, page, start, rows", [
    (H4, BF, 16, [0], [1]), (H4, F32, 16, [0], [1]), (H8, BF, 32, [5], [3]), (H8, F32, 32, [15, 16, 31], [1, 2, 17]), (H7, BF, 256, [0, 300, 0], [0, 9, 1]),
    (H1, BF, 64, [100, 0, 63, 64], [30, 70, 1, 0]), (H1, F32, 128, [127, 0], [2, 40]),
])
@pytest.mark.parametrize("norm, rope", [(True, True), (False, False)])
def test_append(heads, dtype, page, start, rows, norm, rope):
    s = Setup(heads, dtype, page, start, rows, seed=3, norm=norm, rope=rope)
    c = s.cache()
    c.append(s.qkv.to(DEV), ints(s.cu), ints(s.pos + [-1] * (s.room - s.total)), ints(s.slots + [-1] * (s.room - s.total), torch.int64), k_norm=s.dev(s.gain), rope=s.dev(s.rope), eps=pu.EPS)
    x = s.qkv[:s.total].double().view(s.total, -1, s.hd)
    want, mag = pu.normed_rotated(x[:, s.nq:s.nq + s.nkv], s.gain, s.rope, torch.tensor(s.pos))
    slot = torch.tensor(s.slots)
    got_k, got_v = s.kd.cpu(), s.vd.cpu()
    k, v = got_k[slot // page, :, slot % page].double(), got_v[slot // page, :, slot % page]
    # the norm's sum of hd squares, its root and the products with gain, angles and scale: hd + 10 roundings of the terms at most, then one to the type
    assert ((k - want).abs() <= want.abs() * pu.HALF[dtype] + mag * (s.hd + 10) * pu.U32).all()
    assert torch.equal(v, s.qkv[:s.total].view(s.total, -1, s.hd)[:, s.nq + s.nkv:].to(dtype))
    touched = torch.zeros(s.n_pages, page, dtype=torch.bool)
    touched[slot // page, slot % page] = True
    for got, was in ((got_k, s.k), (got_v, s.v)):                 # every other place is as it was, bit for bit
        a, b = got.transpose(1, 2)[~touched], was.transpose(1, 2)[~touched]
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_append_leaves_out_bad_places():
    s = Setup(H4, BF, 16, [3, 0], [4, 2])
    c, n = s.cache(), s.n_pages * 16
    pad = s.room - s.total
    slots = [n, -1, s.slots[2], -(1 << 40), 1 << 40, s.slots[5]]
    pos = [s.pos[0], s.pos[1], -1, s.pos[3], s.pos[4], s.width * 16]         # two more rows with positions beyond the tables
    c.append(s.qkv.to(DEV), ints(s.cu), ints(pos + [0] * pad), ints(slots + [0] * pad, torch.int64), k_norm=s.dev(s.gain), rope=s.dev(s.rope))
    torch.cuda.synchronize()
    for got, was in ((s.kd, s.k), (s.vd, s.v)):
        assert torch.equal(got.cpu().view(torch.int16), was.view(torch.int16))


ATTENTION = [
    # single tokens: one key, a page's end and start, several pages
    (H8, 16, [0], [1]), (H8, 16, [15], [1]), (H8, 16, [16], [1]), (H4, 64, [63, 64, 0, 200, 1], [1, 1, 1, 1, 1]), (H7, 32, [77, 0, 1000], [1, 1, 1]),
    (H16, 128, [500, 3], [1, 1]), (H1, 256, [255, 256, 257], [1, 1, 1]), (H6, 16, [2049], [1]),
    # requests without rows, at the ends and between
    (H8, 32, [40, 50, 60, 70], [0, 2, 0, 1]), (H8, 32, [40, 50, 60], [1, 0, 0]),
    # a few rows: refills
    (H8, 64, [100, 1, 700], [3, 2, 4]), (H8, 16, [33], [5]), (H4, 16, [0, 90], [16, 13]), (H16, 32, [64, 5], [2, 3]), (H7, 16, [61, 200], [7, 3]),
    # several groups of a request's rows, each over several key ranges; ranges of several rounds of a block's waves
    (H4, 16, [1000, 2000], [20, 30]), (H16, 32, [1500], [4]), (H8, 16, [1100, 700], [16, 9]), (H4, 16, [3000] * 40, [1] * 40), (H8, 64, [2500] * 20, [2] * 20),
    # chunks, from the start and behind keys; beside single tokens
    (H8, 64, [0], [130]), (H4, 16, [0, 7], [65, 1]), (H6, 32, [300], [97]), (H7, 256, [130, 0], [75, 40]), (H8, 128, [513, 90, 0, 1100], [200, 1, 1, 1]), (H1, 16, [31], [200]),
    (H16, 64, [20], [40]),
    # long
    (H8, 64, [6000], [1]), (H8, 16, [5000, 10], [3, 1]), (H4, 256, [4000], [70]),
]


@pytest.mark.parametrize("heads, page, start, rows", ATTENTION)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention(heads, page, start, rows, dtype):
    Setup(heads, dtype, page, start, rows, seed=len(start) + sum(rows)).check()


def test_more_groups_than_a_grid_dimension_holds():
    Setup((16, 1, 64), F32, 64, [0] * 128, [640] * 127 + [3], seed=22).check()


def test_ranges_longer_than_a_wave_keeps_page_numbers_for():
    Setup((128, 128, 64), BF, 16, [8999], [1], seed=21).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("norm, rope", [(True, False), (False, True), (False, False)])
def test_attention_without_norm_or_rotation(dtype, norm, rope):
    Setup(H8, dtype, 32, [70, 0, 200], [1, 40, 3], seed=5, norm=norm, rope=rope).check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_scores(dtype):
    """Queries a hundred times as long: nearly all weight on one key, scores far below it underflow."""
    Setup(H8, dtype, 16, [300, 40], [1, 90], seed=6, norm=False, spread=100.0).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [[1, 1], [3, 2], [90, 40]])
def test_pages_apart_and_wide_rows(dtype, rows):
    """K and V interleaved in one allocation, rows of qkv and of out wider than what they hold."""
    s = Setup(H8, dtype, 32, [100, 7], rows, seed=8)
    both = torch.full((s.n_pages, 2) + s.k.shape[1:], float("nan"), dtype=dtype, device=DEV)
    both[:, 0], both[:, 1] = s.k.to(DEV), s.v.to(DEV)
    c = s.cache(kv=(both[:, 0], both[:, 1]))
    wide = torch.full((s.room, s.qkv.shape[1] + 12), float("nan"), device=DEV)
    wide[:, :s.qkv.shape[1]] = s.qkv.to(DEV)
    out = torch.full((s.room, s.nq + 1, s.hd), 5.0, dtype=dtype, device=DEV)
    c.attention(wide[:, :s.qkv.shape[1]], ints(s.start), ints(s.cu), out[:, :s.nq], q_norm=s.dev(s.gain), rope=s.dev(s.rope))
    assert (out[:, s.nq] == 5.0).all() and (out[s.total:] == 5.0).all()
    s.check(out[:s.total, :s.nq].cpu())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("start, rows", [([20], [5]), ([0, 100], [1, 3]), ([0], [90]), ([70, 30], [130, 1])])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf")])
def test_later_values_that_are_not_finite(dtype, start, rows, bad):
    """The newest token's value (and the one's in the middle of a chunk) is not finite: the rows before it come out as if it were finite, those that see it do not."""
    s = Setup(H8, dtype, 16, start, rows, seed=9)
    s.check()
    mid = rows[0] - 1 - rows[0] // 3
    for i, j in ((0, mid), (len(rows) - 1, rows[-1] - 1)):
        p = start[i] + j
        s.v[s.table[i][p // 16], :, p % 16, 3] = bad
    got = s.attend()
    clean = Setup(H8, dtype, 16, start, rows, seed=9)
    ref, tol = clean.reference()
    for i in range(len(rows)):
        first = {0: mid}.get(i, rows[i]) if i == 0 else rows[i]
        if i == len(rows) - 1:
            first = min(first, rows[i] - 1)
        a, b = s.cu[i], s.cu[i] + first
        assert ((got[a:b].double() - ref[a:b]).abs() <= tol[a:b]).all()
        assert not torch.isfinite(got[b:s.cu[i + 1], :, 3]).any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [[1, 1, 1], [4, 3, 2], [100, 70, 33]])
def test_missing_pages(dtype, rows):
    """Pages outside the pool are left out; a row that is left without keys comes out as 0."""
    s = Setup(H8, dtype, 16, [80, 40, 0], rows, seed=10)
    s.table[0][1], s.table[0][3] = -1, s.n_pages
    s.table[1][0] = 1 << 30
    s.table[2] = [-1] * s.width
    ref, tol = s.reference()
    assert (ref[s.cu[2]:] == 0).all()
    s.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_lengths_that_do_not_fit_are_left_out(dtype):
    s = Setup(H8, dtype, 16, [30, 20, 50, 10], [2, 3, 40, 1], seed=11)
    c, ref = s.cache(), s.reference()
    good = s.attend(c)
    s.check(good)

    def run(start, cu, max_new=0):
        out = torch.full((s.room, s.nq, s.hd), 77.0, dtype=dtype, device=DEV)
        c.attention(s.qkv.to(DEV), ints(start), ints(cu), out, q_norm=s.dev(s.gain), rope=s.dev(s.rope), max_new=max_new)
        return out.cpu()

    limit = s.width * 16
    for start, cu, max_new, skipped in [
        ([30, -1, 50, 10], s.cu, 0, [1]), ([30, limit - 2, 50, 10], s.cu, 0, [1]), ([30, 1 << 30, 50, 10], s.cu, 0, [1]), ([30, 20, 50, 10], s.cu, 5, [2]),
        ([30, 20, 50, 10], s.cu[:4] + [s.room + 1], 0, [3]), ([30, 20, 50, 10], s.cu[:4] + [1 << 30], 0, [3]),
    ]:
        out = run(start, cu, max_new)
        for i in range(4):
            a, b = s.cu[i], s.cu[i + 1]
            if i in skipped:
                assert (out[a:b] == 77.0).all(), (start, i)
            else:
                assert torch.equal(out[a:b], good[a:b])
    run([30, 20, 50, 10], [0, 5, 2, -7, 1 << 29])      # not ascending: no access out of range, nothing else is promised
    torch.cuda.synchronize()


@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 2, 1], [100, 1, 2]])
def test_pages_beyond_32_bit_offsets(rows):
    """Pages 2^28 elements apart: those from number 8 on lie beyond 2^31 elements, from 16 on beyond 2^32."""
    s = Setup((4, 2, 64), BF, 16, [100, 60, 130], rows, seed=12)
    gap = 1 << 28
    keep, kv = [], []
    for src in (s.k, s.v):
        flat = torch.empty((s.n_pages - 1) * gap + src[0].numel(), dtype=BF, device=DEV)
        t = flat.as_strided(src.shape, (gap, 16 * 64, 64, 1))
        t.copy_(src.to(DEV))
        keep.append(flat)
        kv.append(t)
    assert s.n_pages > 17 and max(max(r) for r in s.table) >= 17
    c = s.cache(kv=tuple(kv))
    s.check(s.attend(c))
    c.append(s.qkv.to(DEV), ints(s.cu), ints(s.pos + [-1] * (s.room - s.total)), ints(s.slots + [-1] * (s.room - s.total), torch.int64), k_norm=s.dev(s.gain), rope=s.dev(s.rope))
    slot = torch.tensor(s.slots, device=DEV)
    x = s.qkv[:s.total].view(s.total, -1, 64)[:, 6:].to(BF)
    assert torch.equal(kv[1][slot // 16, :, slot % 16].cpu(), x)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_requests(dtype):
    rng = np.random.RandomState(3)
    for n in (65, 300, 1100):
        Setup(H4, dtype, 16, rng.randint(0, 40, n).tolist(), rng.randint(0, 3, n).tolist(), seed=n).check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_requests_of_all_kinds(dtype):
    """More than a wave's lanes of them: single tokens, refills and chunks, behind short and long contexts, each over several key ranges."""
    rng = np.random.RandomState(5)
    start, rows = rng.randint(0, 700, 90), rng.randint(0, 5, 90)
    start[[7, 50, 88]], rows[[7, 50, 88]] = [0, 900, 2100], [150, 77, 130]
    s = Setup(H4, dtype, 32, start.tolist(), rows.tolist(), seed=23)
    s.check()
    assert torch.equal(s.attend(max_new=150), s.attend())


def test_same_bits_every_time_and_on_every_stream():
    s = Setup(H8, BF, 64, [3000, 10, 0, 500], [1, 90, 1, 5], seed=13)
    c = s.cache()
    first = s.attend(c)
    side = torch.cuda.Stream()
    for turn in range(6):
        with torch.cuda.stream(side if turn % 2 else torch.cuda.current_stream()):
            assert torch.equal(s.attend(c), first)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_steps_without_rows(dtype):
    """A step that was refused, and one in which no request brings anything: nothing is stored, nothing comes out."""
    s = Setup(H8, dtype, 16, [20, 3], [4, 1], seed=32)
    c = s.cache()
    tables = pkg.PageTables.empty(1, 16, 2, s.width, DEV)
    for rows, status in (([9, 1], -3), ([0, 0], 0)):
        m = Maps(2, s.room)
        tables.build(ints([0, 0]), ints(rows), *m.all())
        out = torch.full((s.room, s.nq, s.hd), 7.0, dtype=dtype, device=DEV)
        c.append(s.qkv.to(DEV), m.cu, m.pos, m.slots, k_norm=s.dev(s.gain), rope=s.dev(s.rope))
        c.attention(s.qkv.to(DEV), ints([0, 0]), m.cu, out, q_norm=s.dev(s.gain), rope=s.dev(s.rope))
        assert m.status[0].item() == status and m.cu.tolist() == [0, 0, 0]
        assert (out == 7.0).all()
        for got, was in ((s.kd, s.k), (s.vd, s.v)):
            assert torch.equal(got.cpu().view(torch.int16), was.view(torch.int16))


def test_layers_share_a_block_table_and_a_workspace():
    """Handles of several layers one after the other on a stream, and what they refuse."""
    layers = [Setup(H8, BF, 32, [700, 0, 90], [1, 130, 3], seed=30) for _ in range(3)]
    for i, s in enumerate(layers[1:], 1):          # the same tables, other keys and values
        gen = torch.Generator().manual_seed(i)
        for t in (s.k, s.v):
            fresh = torch.randn(t.shape, generator=gen).to(BF)
            t.copy_(torch.where(torch.isnan(t), t, fresh))
    first = layers[0].cache()
    handles = [first] + [first.layer(s.k.to(DEV), s.v.to(DEV)) for s in layers[1:]]
    for _ in range(2):
        for s, c in zip(layers, handles):
            s.check(s.attend(c))
    with pytest.raises(ValueError):
        first.layer(layers[0].kd[:, :1].contiguous(), layers[0].vd)
    with pytest.raises(pkg.DmtdError):
        first.layer(layers[0].kd[:, :, :24].contiguous(), layers[0].vd[:, :, :24].contiguous())


def test_layers_of_other_types_share_a_workspace():
    """Pools of another type behind the same block table; the bfloat16 layer leaves partial results, and the float32 one has more groups in several key ranges than the other can count."""
    layers = [Setup(H8, dtype, 32, [2000] + [300] * 150, [1] * 151, seed=33) for dtype in (BF, F32)]
    first = layers[0].cache()
    handles = [first, first.layer(layers[1].k.to(DEV), layers[1].v.to(DEV))]
    for _ in range(2):
        for s, c in zip(layers, handles):
            s.check(s.attend(c))


def test_the_handles_check_their_tensors():
    s = Setup(H8, BF, 32, [40], [3], seed=31)
    c = s.cache()
    qkv, start, cu, out = s.qkv.to(DEV), ints(s.start), ints(s.cu), torch.zeros(s.room, 8, 128, dtype=BF, device=DEV)
    pos, slots, gain, rope = ints(s.pos + [0] * (s.room - s.total)), ints(s.slots + [0] * (s.room - s.total), torch.int64), s.dev(s.gain), s.dev(s.rope)
    for bad in (dict(qkv=qkv.bfloat16()), dict(qkv=qkv[:-1]), dict(qkv=qkv[:, :1000]), dict(qkv=qkv.t()), dict(start=start.long()), dict(start=ints([1, 2])), dict(cu=cu[:1]),
                dict(cu=cu.cpu()), dict(out=out.float()), dict(out=out[:, :4]), dict(out=out[:2]), dict(q_norm=gain.float()), dict(q_norm=gain[:64]), dict(rope=rope.double()),
                dict(rope=rope[:, :32])):
        a = dict(dict(qkv=qkv, start=start, cu=cu, out=out, q_norm=gain, rope=rope), **bad)
        with pytest.raises(ValueError):
            c.attention(a["qkv"], a["start"], a["cu"], a["out"], q_norm=a["q_norm"], rope=a["rope"])
    for bad in (dict(qkv=qkv[:, :1400]), dict(pos=pos[:-1]), dict(pos=pos.long()), dict(slots=slots.int()), dict(slots=slots[::2])):
        a = dict(dict(qkv=qkv, cu=cu, pos=pos, slots=slots), **bad)
        with pytest.raises(ValueError):
            c.append(a["qkv"], a["cu"], a["pos"], a["slots"], k_norm=gain, rope=rope)
    with pytest.raises(pkg.DmtdError):             # rows that are not 16-byte aligned
        c.attention(torch.zeros(s.room, qkv.shape[1] + 1, device=DEV)[:, 1:], start, cu, out)
    with pytest.raises(pkg.DmtdError):
        c.attention(qkv, start, cu, out, max_new=s.room + 1)
    with pytest.raises(ValueError):
        pkg.PagedCache(s.kd.transpose(1, 2), s.vd.transpose(1, 2), c.block_table, 8, 8)
    with pytest.raises(ValueError):
        pkg.PagedCache(s.kd, s.vd.float(), c.block_table, 8, 8)
    with pytest.raises(pkg.DmtdError):
        pkg.PagedCache(s.kd, s.vd, c.block_table, 7, 8)
    t = pkg.PageTables.empty(8, 16, 2, 4, DEV)
    m = Maps(2, 16)
    for bad in ((start, start) + m.all(), (ints([0, 0]).long(), ints([0, 0])) + m.all(), (ints([0, 0]), ints([0, 0]), m.cu, m.pos, m.slots[:8], m.status)):
        with pytest.raises(ValueError):
            t.build(*bad)
    assert c.attention(qkv, start, cu, q_norm=gain, rope=rope).shape == (s.room, 8, 128)


# ------------------------------------------------------------------------------------------ together

def serve(heads, dtype, page, n_pages, n_req, max_pages, room, lengths, graph):
    """A small server: requests arrive, bring a prompt in chunks, then tokens one by one, and end.  Every step's outputs against the plain form over the
    requests' own keys and values."""
    nq, nkv, hd = heads
    rng, gen = np.random.RandomState(4), torch.Generator().manual_seed(4)
    tables = pkg.PageTables.empty(n_pages, page, n_req, max_pages, DEV)
    nan = torch.full((n_pages, nkv, page, hd), float("nan"), dtype=dtype, device=DEV)
    cache = pkg.PagedCache(nan, nan.clone(), tables.block_table, nq, room)
    gain_q, gain_k = [(1 + 0.2 * torch.randn(hd, generator=gen)).to(dtype) for _ in range(2)]
    rope = pu.rope_table(max_pages * page, hd)
    start_d, rows_d, m = ints([0] * n_req), ints([0] * n_req), Maps(n_req, room)
    qkv_d, out_d = torch.zeros(room, (nq + 2 * nkv) * hd, device=DEV), torch.zeros(room, nq, hd, dtype=dtype, device=DEV)
    gq, gk, rp = gain_q.to(DEV), gain_k.to(DEV), rope.to(DEV)

    def step():
        tables.build(start_d, rows_d, *m.all())
        cache.append(qkv_d, m.cu, m.pos, m.slots, k_norm=gk, rope=rp)
        cache.attention(qkv_d, start_d, m.cu, out_d, q_norm=gq, rope=rp)

    g = None
    if graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
    cached, keys, values = [0] * n_req, [None] * n_req, [None] * n_req
    for turn in range(14):
        rows = []
        for i in range(n_req):
            if cached[i] and rng.rand() < 0.15:
                cached[i], keys[i], values[i] = 0, None, None
                rows.append(0)
            elif cached[i] == 0:
                rows.append(int(rng.choice(lengths)) if rng.rand() < 0.7 else 0)
            else:
                rows.append(int(rng.randint(0, 4)))
            if cached[i] + rows[i] > max_pages * page or sum(rows) > room:
                rows[i] = 0
        total = sum(rows)
        qkv = torch.randn(room, qkv_d.shape[1], generator=gen)
        qkv_d.copy_(qkv)
        out_d.fill_(3.0)
        start_d.copy_(ints(cached))
        rows_d.copy_(ints(rows))
        g.replay() if g else step()
        torch.cuda.synchronize()
        assert m.status.tolist() == [0, 0] and m.cu[-1].item() == total
        at = 0
        got = out_d.cpu()
        for i, r in enumerate(rows):
            if r == 0:
                continue
            x = qkv[at:at + r].view(r, -1, hd)
            pos = torch.arange(cached[i], cached[i] + r)
            k, _ = pu.normed_rotated(x[:, nq:nq + nkv].double(), gain_k, rope, pos)
            new_k, new_v = k.to(dtype), x[:, nq + nkv:].to(dtype)
            keys[i] = new_k if keys[i] is None else torch.cat([keys[i], new_k])
            values[i] = new_v if values[i] is None else torch.cat([values[i], new_v])
            n = keys[i].shape[0]
            # one page of n keys; the cache's own keys may have been rounded to the other neighbour: half a step each, as the queries' own rounding
            ref, tol = pu.attention(x[:, :nq].reshape(r, -1), nq, keys[i].transpose(0, 1)[None], values[i].transpose(0, 1)[None], [[0]], n, [cached[i]], [r], gain_q, rope, dtype is BF)
            q, mag = pu.normed_rotated(x[:, :nq].double(), gain_q, rope, pos)
            slack = 2 * pu.HALF[dtype] * (mag.norm(dim=-1).max() * keys[i].double().norm(dim=-1).max()) / hd ** 0.5 * 2.0 ** -4
            size = values[i].double().abs().max()
            assert ((got[at:at + r].double() - ref).abs() <= tol + slack * size).all()
            cached[i] += r
            at += r
        assert (got[total:] == 3.0).all()


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("heads, dtype, page", [(H8, BF, 16), (H4, F32, 32), (H7, BF, 64)])
def test_the_operators_together(heads, dtype, page, graph):
    serve(heads, dtype, page, 400 * 16 // page, 6, 320 // page, 256, [1, 20, 70, 130], graph)
