"""Attention with shared prefixes against the plain 64-bit form of the paged attention (paged_util), and pages that requests share."""
import ctypes as C

import numpy as np
import pytest
import torch

import paged8_util as p8
import paged_util as pu
import paper_2510_11958_amd as pkg
from test_gpu_paged import BF, DEV, F32, H1, H4, H6, H7, H8, H16, Maps, Setup, ints
from test_gpu_paged8 import E8, Setup8

pytestmark = pytest.mark.gpu


def shared_setup(heads, dtype, page, pages, group, own, rows, **kw):
    """A step whose requests' tables start with the same pages where they are of one group: pages[g] of them; own: cached tokens behind the prefix."""
    front = [pages[g] * page if 0 <= g < len(pages) else 0 for g in group]
    start = [f + o for f, o in zip(front, own)]
    s = Setup8(heads, page, start, rows, **kw) if dtype is E8 else Setup(heads, dtype, page, start, rows, **kw)
    first = {}
    for i, g in enumerate(group):
        if 0 <= g < len(pages):
            lead = first.setdefault(g, i)
            s.table[i][:pages[g]] = s.table[lead][:pages[g]]
    s.group, s.pages = list(group), list(pages)
    return s


def build(s, plan, start=None, cu=None, group=None, pages=None):
    plan.build(ints(start or s.start), ints(cu or s.cu), ints(group or s.group), ints(pages or s.pages))


def attend(s, cache=None, plan=None, rope=True, **kw):
    cache = cache or s.cache()
    if plan is None:
        plan = pkg.SharedPlan(cache, len(s.pages))
        build(s, plan, **kw)
    out = torch.full((s.room, s.nq, s.hd), 77.0, dtype=cache.dtype, device=DEV)
    cache.attention_shared(plan, s.qkv.to(DEV), out, q_norm=s.dev(s.gain), rope=s.dev(s.rope), eps=pu.EPS)
    torch.cuda.synchronize()
    assert (out[s.total:] == 77.0).all()
    return out[:s.total].cpu()


TYPES = [BF, E8, F32]
CASES = [
    # heads, page, pages of the groups, group of each request, tokens behind the prefix, rows
    (H8, 16, [1], [0, 0], [0, 0], [1, 1]),                                       # the shortest prefix, nothing behind it
    (H8, 16, [4], [0, 0, 0], [0, 5, 40], [1, 1, 1]),
    (H4, 64, [2], [0] * 8, [3, 0, 64, 65, 1, 200, 0, 9], [1] * 8),
    (H8, 32, [3, 7], [0, 1, 0, 1, 1, 0], [5, 0, 33, 70, 2, 8], [1, 1, 1, 1, 1, 1]),      # two groups, mixed
    (H7, 16, [5, 2], [1, -1, 0, 0, 5, 1, 1 << 30, 0], [5, 90, 0, 3, 77, 12, 4, 31], [1, 2, 1, 3, 1, 1, 2, 1]),      # some of no group
    (H8, 16, [3, 4, 2], [0, 1, 1, -1], [7, 8, 9, 10], [1, 1, 1, 1]),             # a group of one, a group of none
    (H8, 16, [2], [0, 0, 0, 0], [4, 6, 2, 0], [0, 1, 0, 1]),                     # members without rows, the first among them
    (H8, 16, [2, 2], [0, 0, 1, 1], [4, 6, 2, 0], [0, 1, 1, 0]),                  # groups of which one request brings rows
    (H16, 128, [2], [0, 0, 0, 0], [1, 130, 5, 127], [1, 2, 1, 1]),
    (H1, 256, [1], [0, 0, 0], [256, 0, 3], [1, 1, 2]),
    (H6, 16, [30], [0] * 5, [10, 20, 30, 0, 50], [3, 1, 2, 3, 1]),               # a few rows each
    # more rows than the few-rows blocks take, together or alone
    (H8, 16, [6], [0] * 40, list(range(40)), [1] * 40),
    (H8, 64, [5], [0] * 3, [0, 20, 50], [70, 3, 1]),
    (H4, 16, [9, 4], [0, 1] * 4, [2, 3, 100, 0, 5, 8, 1, 30], [30, 1, 50, 2, 1, 80, 1, 1]),
    (H16, 32, [8], [0] * 20, [3] * 20, [2] * 20),
    (H7, 32, [7], [0] * 30, [5] * 30, [1, 2, 1] * 10),
    # prefixes of several key ranges, own keys of several
    (H8, 64, [50], [0] * 6, [0, 100, 700, 3, 1500, 20], [1, 1, 1, 1, 1, 1]),
    (H8, 16, [130], [0] * 24, [9] * 24, [3] * 24),
    (H4, 32, [60, 100], [0, 1, 1, 0, 1, 0], [1000, 0, 2000, 5, 70, 80], [20, 1, 40, 90, 3, 1]),
    (H8, 64, [80], [0, 0, 0], [40, 0, 300], [150, 200, 1]),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("dtype", TYPES)
def test_shared_attention(case, dtype):
    heads, page, pages, group, own, rows = CASES[case]
    s = shared_setup(heads, dtype, page, pages, group, own, rows, seed=case)
    s.check(attend(s))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("norm, rope", [(True, False), (False, True), (False, False)])
def test_without_norm_or_rotation(dtype, norm, rope):
    s = shared_setup(H8, dtype, 32, [4], [0, 0, -1, 0], [5, 0, 40, 17], [1, 40, 1, 3], seed=5, norm=norm, rope=rope)
    s.check(attend(s))


@pytest.mark.parametrize("dtype", TYPES)
def test_large_scores(dtype):
    s = shared_setup(H8, dtype, 16, [20], [0] * 4, [30, 0, 100, 5], [1, 90, 1, 2], seed=6, norm=False, spread=100.0)
    s.check(attend(s))


@pytest.mark.parametrize("dtype", TYPES)
def test_groups_that_do_not_fit_go_by_themselves(dtype):
    """Prefixes of no pages, negative ones, ones beyond the table or beyond a request's cached tokens: the results are those of the requests' own tables."""
    s = shared_setup(H8, dtype, 16, [4, 3], [0, 0, 1, 1, 0], [2, 10, 0, 7, 3], [1, 2, 1, 1, 3], seed=7)
    good = attend(s)
    s.check(good)
    for pages in ([0, 3], [-1, 0], [1 << 30, 3], [s.width + 1, -(1 << 31)], [4, 4], [5, 3], [2147483647, 2]):
        s.check(attend(s, pages=pages))
    for group in ([9, 9, 9, 9, 9], [-1] * 5, [-(1 << 31), 2, 1, 1, 0]):
        s.check(attend(s, group=group))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_requests(dtype):
    rng = np.random.RandomState(3)
    for n, groups in ((63, 2), (65, 40), (300, 3), (1100, 300)):
        pages = rng.randint(1, 5, groups).tolist()
        s = shared_setup(H4, dtype, 16, pages, rng.randint(-1, groups, n).tolist(), rng.randint(0, 40, n).tolist(), rng.randint(0, 3, n).tolist(), seed=n)
        s.check(attend(s))
    start, rows = rng.randint(0, 300, 90), rng.randint(0, 5, 90)
    start[[7, 50, 88]], rows[[7, 50, 88]] = [0, 500, 900], [150, 77, 130]
    s = shared_setup(H4, dtype, 32, [20, 9], rng.randint(-1, 2, 90).tolist(), start.tolist(), rows.tolist(), seed=23, room=2048)
    s.check(attend(s))


@pytest.mark.parametrize("dtype", TYPES)
def test_more_groups_than_requests(dtype):
    s = shared_setup(H4, dtype, 16, [2] * 500, [499, 3, 499, 3], [1, 2, 3, 4], [1, 1, 1, 2], seed=24)
    s.check(attend(s))


@pytest.mark.parametrize("dtype", TYPES)
def test_ranges_longer_than_a_wave_keeps_page_numbers_for(dtype):
    """64 KV heads leave each of them 16 ranges: of a prefix of 20000 tokens a wave's have 1280 keys, 80 groups of 16."""
    s = shared_setup((64, 64, 64), dtype, 16, [1250], [0, 0], [3, 40], [1, 1], seed=25)
    s.check(attend(s))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_long_prefix(dtype):
    """One KV head and 130 thousand shared tokens, behind them rows of a block's tile and more."""
    s = shared_setup((4, 1, 64), dtype, 256, [512], [0, 0, -1, 0], [7, 300, 50, 0], [1, 2, 1, 40], seed=26)
    s.check(attend(s))


def test_as_many_requests_and_groups_as_there_can_be():
    """8192 of either, whose tables lie in memory instead of LDS, most of the groups of three requests, and rows beyond one round of the join."""
    n = 8192
    rng = np.random.RandomState(7)
    s = shared_setup((2, 1, 64), BF, 16, [1] * n, rng.permutation(np.arange(n) % 2731).tolist(), rng.randint(0, 20, n).tolist(), (rng.rand(n) < 0.7).astype(int).tolist(), seed=27)
    s.check(attend(s))


def test_many_rows_in_groups():
    """Chunks of thousands of rows behind a shared prefix: more tiles than blocks, more rows than the join's grid."""
    s = shared_setup((4, 2, 64), BF, 32, [3], [0, 0, 0], [0, 50, 7], [2500, 1, 1700], seed=28)
    s.check(attend(s))


def test_two_plans_at_once():
    """Two steps of the same caches on two streams, eager and replayed from two graphs in turn, each with its plan and output."""
    steps = [shared_setup(H8, BF, 16, [40, 3], [0, 1, 0, 0, -1, 1], [5, 60, 0, 700, 30, 2], rows, seed=29) for rows in ([1, 2, 1, 1, 3, 1], [30, 1, 1, 60, 1, 2])]
    want, runs = [], []
    for s in steps:
        c = s.cache()
        plan = pkg.SharedPlan(c, 2)
        args = [ints(s.start), ints(s.cu), ints(s.group), ints(s.pages)]
        qkv, out, gain, rope = s.qkv.to(DEV), torch.zeros(s.room, s.nq, s.hd, dtype=BF, device=DEV), s.dev(s.gain), s.dev(s.rope)

        def run(c=c, plan=plan, args=args, qkv=qkv, out=out, gain=gain, rope=rope):
            plan.build(*args)
            c.attention_shared(plan, qkv, out, q_norm=gain, rope=rope, eps=pu.EPS)
            return out

        s.check(run()[:s.total].cpu())
        want.append(run().clone())
        runs.append(run)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(5):
        for st, run in zip(streams, runs):
            with torch.cuda.stream(st):
                run().zero_()
                run()
    torch.cuda.synchronize()
    for run, w in zip(runs, want):
        assert torch.equal(run(), w)
    graphs = []
    for st, run in zip(streams, runs):
        st.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            out = run()
        graphs.append((g, out))
    for turn in range(6):
        for g, out in graphs:
            out.zero_()
            g.replay()
        torch.cuda.synchronize()
        for (g, out), w in zip(graphs, want):
            assert torch.equal(out, w), turn


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [[1, 1, 1], [4, 3, 2], [100, 70, 33]])
def test_missing_pages(dtype, rows):
    """Pages outside the pool, in the prefix and behind it, are left out; rows that are left without keys come out as 0."""
    s = shared_setup(H8, dtype, 16, [3, 1], [0, 0, 1, 1], [20, 40, 0, 0], rows + [1], seed=10)
    for i in (0, 1):
        s.table[i][1] = -1
    s.table[0][4], s.table[1][3] = s.n_pages, 1 << 30
    s.table[2] = s.table[3] = [-1] * s.width
    ref, _ = s.reference()
    assert (ref[s.cu[2]:] == 0).all()
    s.check(attend(s))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [[2, 1, 3], [90, 1, 40]])
def test_values_that_are_not_finite(dtype, rows):
    """Of the newest token, which only its own row sees, and in the prefix, which all rows of the group see and no others."""
    s = shared_setup(H8, dtype, 16, [4], [0, 0, -1], [20, 0, 30], rows, seed=9)
    ref, tol = s.reference()
    last = s.start[0] + rows[0] - 1

    def spoil(t, i, p):
        if dtype is E8:
            t[s.table[i][p // 16], :, p % 16, 3] = 0x7F
        else:
            t[s.table[i][p // 16], :, p % 16, 3] = float("nan")

    spoil(s.vb if dtype is E8 else s.v, 0, last)
    got = attend(s)
    rest = torch.ones(s.total, dtype=torch.bool)
    rest[rows[0] - 1] = False
    assert ((got.double() - ref).abs() <= tol)[rest].all()
    assert torch.isnan(got[rows[0] - 1, :, 3]).all()
    spoil(s.vb if dtype is E8 else s.v, 1, 37)
    got = attend(s)
    assert ((got.double() - ref).abs() <= tol)[s.cu[2]:].all()
    assert torch.isnan(got[:s.cu[2], :, 3]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_that_do_not_fit_are_left_out(dtype):
    s = shared_setup(H8, dtype, 16, [2], [0, 0, 0, -1], [30, 20, 50, 10], [2, 3, 40, 1], seed=11)
    c = s.cache()
    good = attend(s, c)
    s.check(good)
    ref, tol = s.reference()
    limit = s.width * 16
    for start, cu, skipped in [([62, -1, 82, 10], s.cu, 1), ([62, limit - 2, 82, 10], s.cu, 1), ([62, 1 << 30, 82, 10], s.cu, 1), ([62, 52, 82, 10], s.cu[:4] + [s.room + 1], 3)]:
        plan = pkg.SharedPlan(c, 1)
        build(s, plan, start=start, cu=cu)
        out = torch.full((s.room, s.nq, s.hd), 77.0, dtype=c.dtype, device=DEV)
        c.attention_shared(plan, s.qkv.to(DEV), out, q_norm=s.dev(s.gain), rope=s.dev(s.rope))
        out = out.cpu()
        for i in range(4):
            a, b = s.cu[i], s.cu[i + 1]
            if i == skipped:
                assert (out[a:b] == 77.0).all(), (start, i)
            else:      # (the ranges may be others without the one that is left out)
                assert ((out[a:b].double() - ref[a:b]).abs() <= tol[a:b]).all()
        assert (out[s.total:] == 77.0).all()
    plan = pkg.SharedPlan(c, 1)
    build(s, plan, cu=[0, 5, 2, 7, 8])      # not ascending: no rows at all
    assert (attend(s, c, plan) == 77.0).all()
    build(s, plan)
    assert torch.equal(attend(s, c, plan), good)


def test_a_plan_that_was_not_built_or_is_of_another_layout():
    s = shared_setup(H8, BF, 16, [2], [0, 0], [3, 4], [1, 2], seed=12)
    c = s.cache()
    plan = pkg.SharedPlan(c, 1)
    assert (attend(s, c, plan) == 77.0).all()
    build(s, plan)
    s.check(attend(s, c, plan))
    other = pkg.PagedCache(s.kd, s.vd, c.block_table, s.nq, s.room - 1)
    with pytest.raises(ValueError):
        attend(s, other, plan)
    # the library itself, which cannot see what the memory was built for: nothing is written
    lib = pkg.load_library()
    out = torch.full((s.room, s.nq, s.hd), 77.0, dtype=BF, device=DEV)
    qkv = s.qkv.to(DEV)
    rc = lib.dmtd_paged_attention_shared(other._p, plan._p, qkv.data_ptr(), qkv.shape[1], None, 0.0, None, 0, out.data_ptr(), s.nq * s.hd, 0)
    torch.cuda.synchronize()
    assert rc == 0 and (out == 77.0).all()


def test_positions_without_angles_are_left_out():
    """A plan for fewer positions than the table has places: requests beyond them are left out, and the rotary table may be that short."""
    s = shared_setup(H8, BF, 16, [2], [0, 0, 0], [0, 20, 60], [1, 2, 3], seed=15)
    c = s.cache()
    ref, tol = s.reference()
    plan = pkg.SharedPlan(c, 1, positions=80)
    build(s, plan)
    out = torch.full((s.room, s.nq, s.hd), 77.0, dtype=BF, device=DEV)
    c.attention_shared(plan, s.qkv.to(DEV), out, q_norm=s.dev(s.gain), rope=s.dev(s.rope[:80].contiguous()))
    got = out.cpu()
    assert ((got[:3].double() - ref[:3]).abs() <= tol[:3]).all() and (got[3:] == 77.0).all()
    with pytest.raises(pkg.DmtdError):
        c.attention_shared(plan, s.qkv.to(DEV), out, rope=s.dev(s.rope[:79].contiguous()))
    full = pkg.SharedPlan(c, 1)
    build(s, full)
    with pytest.raises(pkg.DmtdError):
        c.attention_shared(full, s.qkv.to(DEV), out, rope=s.dev(s.rope[:80].contiguous()))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 2, 90]])
def test_pages_apart_and_wide_rows(dtype, rows):
    s = shared_setup(H8, dtype, 32, [3], [0, 0, 0], [100, 7, 30], rows, seed=8)
    both = torch.full((s.n_pages, 2) + s.k.shape[1:], float("nan"), dtype=dtype, device=DEV)
    both[:, 0], both[:, 1] = s.k.to(DEV), s.v.to(DEV)
    c = s.cache(kv=(both[:, 0], both[:, 1]))
    wide = torch.full((s.room, s.qkv.shape[1] + 12), float("nan"), device=DEV)
    wide[:, :s.qkv.shape[1]] = s.qkv.to(DEV)
    out = torch.full((s.room, s.nq + 1, s.hd), 5.0, dtype=dtype, device=DEV)
    plan = pkg.SharedPlan(c, 1)
    build(s, plan)
    c.attention_shared(plan, wide[:, :s.qkv.shape[1]], out[:, :s.nq], q_norm=s.dev(s.gain), rope=s.dev(s.rope))
    assert (out[:, s.nq] == 5.0).all() and (out[s.total:] == 5.0).all()
    s.check(out[:s.total, :s.nq].cpu())


@pytest.mark.parametrize("rows", [[1, 1, 1], [100, 1, 2]])
def test_pages_beyond_32_bit_offsets(rows):
    s = shared_setup((4, 2, 64), BF, 16, [4], [0, 0, 0], [100, 0, 66], rows, seed=12)
    gap = 1 << 28
    kv = []
    for src in (s.k, s.v):
        t = torch.empty((s.n_pages - 1) * gap + src[0].numel(), dtype=BF, device=DEV).as_strided(src.shape, (gap, 16 * 64, 64, 1))
        t.copy_(src.to(DEV))
        kv.append(t)
    assert max(s.table[1][:4]) >= 8 and max(max(r) for r in s.table) >= 17
    s.check(attend(s, s.cache(kv=tuple(kv))))


def test_same_bits_every_time_and_on_every_stream():
    rng = np.random.RandomState(2)
    s = shared_setup(H8, BF, 64, [30, 4], rng.randint(-1, 2, 40).tolist(), rng.randint(0, 300, 40).tolist(), rng.randint(0, 3, 40).tolist(), seed=13)
    c = s.cache()
    plan = pkg.SharedPlan(c, 2)
    build(s, plan)
    first = attend(s, c, plan)
    s.check(first)
    side = torch.cuda.Stream()
    for turn in range(6):
        with torch.cuda.stream(side if turn % 2 else torch.cuda.current_stream()):
            build(s, plan)
            assert torch.equal(attend(s, c, plan), first)
        torch.cuda.synchronize()


def test_one_plan_serves_layers_of_both_types():
    """A bfloat16 and an 8-bit layer behind one block table; an fp32 one needs a plan of its own."""
    a = shared_setup(H8, BF, 32, [20], [0] * 20, [30] * 20, [1, 2] * 10, seed=30)
    b = shared_setup(H8, E8, 32, [20], [0] * 20, [30] * 20, [1, 2] * 10, seed=30)
    first = a.cache()
    second = first.layer(b.kb.to(DEV).view(E8), b.vb.to(DEV).view(E8), k_scale=b.ke.to(DEV), v_scale=b.ve.to(DEV))
    plan = pkg.SharedPlan(first, 1)
    build(a, plan)
    for _ in range(2):
        a.check(attend(a, first, plan))
        b.check(attend(b, second, plan))
    with pytest.raises(ValueError):
        attend(a, first.layer(a.k.float().to(DEV), a.v.float().to(DEV)), plan)


def test_the_handles_check_their_tensors():
    s = shared_setup(H8, BF, 32, [1, 2], [0, 1], [40, 3], [3, 1], seed=31)
    c = s.cache()
    for n in (0, 8193):
        with pytest.raises(pkg.DmtdError):
            pkg.SharedPlan(c, n)
    with pytest.raises(ValueError):
        pkg.SharedPlan(c, 1, positions=-1)
    plan = pkg.SharedPlan(c, 2)
    start, cu, group, pages = ints(s.start), ints(s.cu), ints(s.group), ints(s.pages)
    for bad in ((start.long(), cu, group, pages), (start, cu[:-1], group, pages), (start, cu, group[:1], pages), (start, cu, group, pages[:1]), (start, cu, group.cpu(), pages),
                (start, cu, group, pages.float())):
        with pytest.raises(ValueError):
            plan.build(*bad)
    plan.build(start, cu, group, pages)
    qkv = s.qkv.to(DEV)
    for bad in (dict(qkv=qkv.bfloat16()), dict(qkv=qkv[:-1]), dict(out=torch.zeros(s.room, 8, 128, device=DEV)), dict(q_norm=torch.zeros(128, device=DEV)), dict(rope=s.rope.double().to(DEV))):
        with pytest.raises(ValueError):
            c.attention_shared(plan, **dict(dict(qkv=qkv), **bad))
    assert c.attention_shared(plan, qkv).shape == (s.room, 8, 128)


# ------------------------------------------------------------------------------------------ pages that requests share

def test_page_tables_leave_shared_pages_alone():
    t = pkg.PageTables.empty(20, 16, 4, 6, DEV)
    m = Maps(4, 128)
    t.build(ints([0, 0, 0, 0]), ints([40, 0, 0, 0]), *m.all(), shared=ints([0, 0, 0, 0]))      # request 0 holds pages 0, 1, 2
    assert t.block_table[0].tolist() == [0, 1, 2, -1, -1, -1] and m.status.tolist() == [0, 0]
    t.block_table[1, :2] = t.block_table[0, :2]                                              # request 1 and 2 stand behind two of them
    t.block_table[2, :2] = t.block_table[0, :2]
    t.held[1:3] = 2
    shared = ints([0, 2, 2, 0])
    t.build(ints([40, 32, 32, 0]), ints([0, 5, 17, 1]), *m.all(), shared=shared)
    assert t.block_table.tolist() == [[0, 1, 2, -1, -1, -1], [0, 1, 3, -1, -1, -1], [0, 1, 4, 5, -1, -1], [6, -1, -1, -1, -1, -1]]
    assert t.held.tolist() == [3, 3, 4, 1] and t.n_free.item() == 13 and m.cu.tolist() == [0, 0, 5, 22, 23]
    assert m.pos[:23].tolist() == list(range(32, 37)) + list(range(32, 49)) + [0]
    assert m.slots[:23].tolist() == [3 * 16 + j for j in range(5)] + [4 * 16 + j for j in range(16)] + [5 * 16, 6 * 16]
    t.build(ints([40, 0, 49, 1]), ints([0, 0, 1, 1]), *m.all(), shared=shared)               # request 1 ends: its own page goes back, the others stay
    assert t.block_table[1].tolist() == [0, 1, -1, -1, -1, -1] and t.held.tolist() == [3, 2, 4, 1] and t.n_free.item() == 14
    assert t.free_pages[13].item() == 3
    was = [x.clone() for x in (t.block_table, t.held, t.free_pages, t.n_free)]
    for bad, who in (([0, 3, 2, 0], 1), ([-1, 2, 2, 0], 0), ([0, 2, 2, 7], 3)):              # more than held, negative
        t.build(ints([40, 0, 49, 1]), ints([0, 0, 1, 1]), *m.all(), shared=ints(bad))
        assert m.status.tolist() == [-1, who] and m.cu.tolist() == [0] * 5
        for a, b in zip(was, (t.block_table, t.held, t.free_pages, t.n_free)):
            assert torch.equal(a, b)
    t.build(ints([0, 0, 0, 0]), ints([0, 0, 0, 0]), *m.all(), shared=shared)                 # all end
    assert t.n_free.item() == 20 and t.held.tolist() == [0, 2, 2, 0] and sorted(t.free_pages.tolist()) == list(range(20))


@pytest.mark.parametrize("n_req, room", [(8, 64), (80, 512), (300, 1024), (300, 4096)])
def test_shared_pages_in_every_layout_of_the_tables(n_req, room):
    """Half of the requests stand behind request 0's pages: what is taken and given back is what they need beyond these."""
    t = pkg.PageTables.empty(6 * n_req + 4, 16, n_req, 10, DEV)
    m = Maps(n_req, room)
    zero = [0] * n_req
    t.build(ints(zero), ints([50] + zero[1:]), *m.all())
    followers = list(range(1, n_req, 2))
    for i in followers:
        t.block_table[i, :3] = t.block_table[0, :3]
        t.held[i] = 3
    shared = ints([3 if i in followers else 0 for i in range(n_req)])
    free = t.n_free.item()
    start = [50] + [48 if i in followers else 0 for i in range(1, n_req)]
    rows = [0] + [1 + i % 3 for i in range(1, n_req)]
    t.build(ints(start), ints(rows), *m.all(), shared=shared)
    assert m.status.tolist() == [0, 0] and t.n_free.item() == free - (n_req - 1)
    assert t.held.tolist() == [4] + [4 if i in followers else 1 for i in range(1, n_req)]
    table = t.block_table.tolist()
    assert all(table[i][:3] == table[0][:3] for i in followers)
    pages = [p for i, r in enumerate(table) for p in (r[3:] if i in followers else r) if p >= 0]
    assert len(set(pages)) == len(pages)
    cu = m.cu.tolist()
    for i in range(n_req):
        for j in range(rows[i]):
            p = start[i] + j
            assert m.pos[cu[i]:cu[i + 1]].tolist()[j] == p and m.slots[cu[i]:cu[i + 1]].tolist()[j] == table[i][p // 16] * 16 + p % 16
        if i > 20:
            break
    t.build(ints([50] + zero[1:]), ints(zero), *m.all(), shared=shared)
    assert t.n_free.item() == free and t.held.tolist() == [4] + [3 if i in followers else 0 for i in range(1, n_req)]


# ------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("heads, dtype, page", [(H8, BF, 16), (H8, E8, 32), (H4, F32, 16), (H7, E8, 16)])
def test_the_operators_together(heads, dtype, page, graph):
    """A small server: request 0 brings a document in chunks, others arrive behind its whole pages, bring questions, get tokens one by one and end, beside one without it.  Every step's
    outputs against the plain form over what the pool holds (read back), and at the end every page is free again."""
    nq, nkv, hd = heads
    n_req, doc, max_pages, room = 7, 5 * page + 9, 320 // page, 256
    n_pages = 80 * 16 // page
    wide = BF if dtype is E8 else dtype
    gen, rng = torch.Generator().manual_seed(4), np.random.RandomState(4)
    tables = pkg.PageTables.empty(n_pages, page, n_req, max_pages, DEV)
    pools = [torch.zeros(n_pages, nkv, page, hd, device=DEV).to(dtype) for _ in range(2)]
    scales = {n: torch.zeros(n_pages, nkv, page, dtype=torch.uint8, device=DEV) for n in ("k_scale", "v_scale")} if dtype is E8 else {}
    cache = pkg.PagedCache(pools[0], pools[1], tables.block_table, nq, room, **scales)
    plan = pkg.SharedPlan(cache, 1)
    gain_q, gain_k = [(1 + 0.2 * torch.randn(hd, generator=gen)).to(wide) for _ in range(2)]
    rope = pu.rope_table(max_pages * page, hd)
    start_d, rows_d, group_d, pages_d, shared_d, m = ints([0] * n_req), ints([0] * n_req), ints([-1] * n_req), ints([doc // page]), ints([0] * n_req), Maps(n_req, room)
    qkv_d, out_d = torch.zeros(room, (nq + 2 * nkv) * hd, device=DEV), torch.zeros(room, nq, hd, dtype=wide, device=DEV)
    gq, gk, rp = gain_q.to(DEV), gain_k.to(DEV), rope.to(DEV)

    def step():
        tables.build(start_d, rows_d, *m.all(), shared=shared_d)
        cache.append(qkv_d, m.cu, m.pos, m.slots, k_norm=gk, rope=rp)
        plan.build(start_d, m.cu, group_d, pages_d)
        cache.attention_shared(plan, qkv_d, out_d, q_norm=gq, rope=rp)

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
    cached, member = [0] * n_req, [False] * n_req
    for turn in range(14):
        rows = [0] * n_req
        if turn < 2:
            rows[0] = doc // 2 if turn == 0 else doc - doc // 2
        else:
            for i in range(1, n_req):
                if member[i] and rng.rand() < 0.2:
                    cached[i], member[i] = 0, False                # its own pages go back in this step
                    continue
                if i < n_req - 1 and not member[i] and tables.held[i].item() == shared_d[i].item():      # arrives
                    tables.block_table[i, :doc // page] = tables.block_table[0, :doc // page]
                    tables.held[i] = shared_d[i] = doc // page
                    cached[i], member[i], rows[i] = doc // page * page, True, int(rng.randint(1, 40))
                elif i == n_req - 1 or member[i]:
                    rows[i] = int(rng.randint(0, 4))
                if cached[i] + rows[i] > max_pages * page or sum(rows) > room:
                    rows[i] = 0
            rows[0] = 1 if turn == 7 else 0                        # the document's own request goes on once
        for i in range(n_req):
            group_d[i] = 0 if member[i] or (i == 0 and turn >= 2) else -1
        total = sum(rows)
        qkv = torch.randn(room, qkv_d.shape[1], generator=gen)
        qkv_d.copy_(qkv)
        out_d.fill_(3.0)
        start_d.copy_(ints(cached))
        rows_d.copy_(ints(rows))
        g.replay() if g else step()
        torch.cuda.synchronize()
        assert m.status.tolist() == [0, 0] and m.cu[-1].item() == total
        table = tables.block_table.tolist()
        everything = torch.arange(n_pages * page, device=DEV)
        k, v = [t.view(n_pages, page, nkv, hd).transpose(1, 2).cpu() for t in cache.read(everything)]
        ref, tol = (p8.attention if dtype is E8 else pu.attention)(qkv, nq, k, v, table, page, cached, rows, gain_q, rope, dtype is not F32)
        got = out_d.cpu()
        assert ((got[:total].double() - ref).abs() <= tol).all(), turn
        assert (got[total:] == 3.0).all()
        cached = [c + r for c, r in zip(cached, rows)]
    start_d.zero_()
    rows_d.zero_()
    group_d.fill_(-1)
    g.replay() if g else step()
    assert tables.n_free.item() == n_pages and sorted(tables.free_pages.tolist()) == list(range(n_pages))
