"""Shared prefixes over 8-bit pools whose pages and scales lie apart, and two plans of one cache at once."""
import pytest
import torch

import paged_util as pu
import paper_2510_11958_amd as pkg
from test_gpu_paged import BF, DEV, H8, ints
from test_gpu_paged8 import E8
from test_gpu_paged_shared import attend, build, shared_setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 2, 90]])
def test_8_bit_pages_apart_and_wide_rows(rows):
    """Codes and scales of K and V interleaved in one allocation each, rows of qkv and of out wider than what they hold."""
    s = shared_setup(H8, E8, 32, [3], [0, 0, 0], [100, 7, 30], rows, seed=8)
    both = torch.full((s.n_pages, 2) + s.kb.shape[1:], 0x7F, dtype=torch.uint8, device=DEV)
    scales = torch.full((s.n_pages, 3) + s.ke.shape[1:], 255, dtype=torch.uint8, device=DEV)
    both[:, 0], both[:, 1], scales[:, 0], scales[:, 1] = s.kb.to(DEV), s.vb.to(DEV), s.ke.to(DEV), s.ve.to(DEV)
    c = s.cache(kv=(both[:, 0], both[:, 1]), scales=(scales[:, 0], scales[:, 1]))
    wide = torch.full((s.room, s.qkv.shape[1] + 12), float("nan"), device=DEV)
    wide[:, :s.qkv.shape[1]] = s.qkv.to(DEV)
    out = torch.full((s.room, s.nq + 1, s.hd), 5.0, dtype=BF, device=DEV)
    plan = pkg.SharedPlan(c, 1)
    build(s, plan)
    c.attention_shared(plan, wide[:, :s.qkv.shape[1]], out[:, :s.nq], q_norm=s.dev(s.gain), rope=s.dev(s.rope))
    assert (out[:, s.nq] == 5.0).all() and (out[s.total:] == 5.0).all()
    s.check(out[:s.total, :s.nq].cpu())


@pytest.mark.parametrize("rows", [[1, 1, 1], [100, 1, 2]])
def test_8_bit_pages_beyond_32_bit_offsets(rows):
    """Pages of codes 2^28 bytes apart and their scales 2^28 too: those from number 8 on lie beyond 2^31, from 16 on beyond 2^32."""
    s = shared_setup((4, 2, 64), E8, 16, [4], [0, 0, 0], [100, 0, 66], rows, seed=12)
    gap = 1 << 28
    far = []
    for src in (s.kb, s.vb, s.ke, s.ve):
        t = torch.empty((s.n_pages - 1) * gap + src[0].numel(), dtype=torch.uint8, device=DEV).as_strided(src.shape, (gap,) + src.stride()[1:])
        t.copy_(src.to(DEV))
        far.append(t)
    assert max(s.table[1][:4]) >= 8 and max(max(r) for r in s.table) >= 17
    s.check(attend(s, s.cache(kv=tuple(far[:2]), scales=tuple(far[2:]))))


@pytest.mark.parametrize("dtype", [BF, E8])
def test_two_plans_of_one_cache_at_once(dtype):
    """Two steps over one pool, through one handle and one block table, on two streams: each with a plan, a workspace, lengths and groups of its own; eager and from two graphs."""
    s = shared_setup(H8, dtype, 16, [40, 3], [0, 1, 0, 0, -1, 1], [5, 60, 0, 700, 30, 2], [30, 2, 5, 60, 3, 2], seed=29)
    c, gain, rope = s.cache(), s.dev(s.gain), s.dev(s.rope)
    # the second step: fewer rows of each request, further in front, in other groups
    steps = [(s.start, s.rows, s.group, s.pages), ([x - 1 for x in s.start], [1, 2, 1, 7, 1, 1], [0, -1, 0, 0, -1, -1], [39, 1])]
    want, runs, outs = [], [], []
    for start, rows, group, pages in steps:
        cu = [0]
        for r in rows:
            cu.append(cu[-1] + r)
        plan = pkg.SharedPlan(c, 2)
        args = [ints(start), ints(cu), ints(group), ints(pages)]
        qkv, out = s.qkv.to(DEV), torch.zeros(s.room, s.nq, s.hd, dtype=BF, device=DEV)

        def run(plan=plan, args=args, qkv=qkv, out=out):
            plan.build(*args)
            c.attention_shared(plan, qkv, out, q_norm=gain, rope=rope, eps=pu.EPS)

        run()
        s.start, s.rows = start, rows
        s.check(out[:sum(rows)].cpu())
        want.append(out.clone())
        runs.append(run)
        outs.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for turn in range(10):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for st, run in zip(streams, runs):
            with torch.cuda.stream(st):
                run()
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert torch.equal(out, w), turn
    graphs = []
    for st, run in zip(streams, runs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            run()
        graphs.append(g)
    for turn in range(6):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert torch.equal(out, w), turn
