"""Refusals of the calls of shared prefixes, from the host's checks, before anything is enqueued.  No GPU needed."""
import ctypes as C

import pytest

import paper_2510_11958_amd as pkg
from paper_2510_11958_amd.binding import _SharedPlan
from test_paged_host import BAD_CACHE, TABLES, P, cache, pool, refused


def plan(**kw):
    a = dict(n_groups=2, positions=0, plan=P, plan_bytes=1 << 40, workspace=P, workspace_bytes=1 << 40)
    a.update(kw)
    return _SharedPlan(*a.values())


BUILD = dict(start=P, cu=P, group=P, prefix_pages=P)
ATTENTION = dict(qkv=P, ld=256, gain=P, eps=1e-6, rope=P, rope_len=64, out=P, ldo=256)
BAD_PLAN = [
    (dict(n_groups=0), "n_groups"), (dict(n_groups=8193), "n_groups"), (dict(positions=-1), "positions"), (dict(plan=None), "plan"), (dict(plan=P + 128), "plan"),
    (dict(workspace=None), "workspace"), (dict(workspace=P + 64), "workspace"),
]


@pytest.mark.parametrize("in_plan, word", BAD_PLAN)
def test_a_bad_plan_is_refused(in_plan, word):
    lib, c, p = pkg.load_library(), cache(), plan(**in_plan)
    refused(lib.dmtd_shared_plan_build(C.byref(c), C.byref(p), *BUILD.values(), None), word)
    refused(lib.dmtd_paged_attention_shared(C.byref(c), C.byref(p), *ATTENTION.values(), None), word)


@pytest.mark.parametrize("in_cache, word", BAD_CACHE)
def test_a_bad_cache_is_refused(in_cache, word):
    lib, c, p = pkg.load_library(), cache(**in_cache), plan()
    refused(lib.dmtd_shared_plan_build(C.byref(c), C.byref(p), *BUILD.values(), None), word)
    refused(lib.dmtd_paged_attention_shared(C.byref(c), C.byref(p), *ATTENTION.values(), None), word)
    assert lib.dmtd_shared_plan_bytes(C.byref(c), 2) == 0 and lib.dmtd_shared_workspace_bytes(C.byref(c)) == 0


@pytest.mark.parametrize("args, word", [(dict(start=None), "start"), (dict(cu=P + 2), "cu_rows"), (dict(group=None), "group"), (dict(prefix_pages=P + 1), "prefix_pages")])
def test_building_a_plan_refuses(args, word):
    refused(pkg.load_library().dmtd_shared_plan_build(C.byref(cache()), C.byref(plan()), *dict(BUILD, **args).values(), None), word)


@pytest.mark.parametrize("args, word", [
    (dict(qkv=None), "qkv"), (dict(qkv=P + 4), "qkv"), (dict(ld=252), "ld"), (dict(gain=P + 8), "gain"), (dict(eps=float("nan")), "eps"), (dict(rope=P + 8), "rotary"),
    (dict(rope_len=0), "rotary"), (dict(rope_len=63), "rotary"), (dict(out=None), "out"), (dict(out=P + 8), "out"), (dict(ldo=248), "ldo"), (dict(ldo=260), "ldo"),
])
def test_shared_attention_refuses(args, word):
    """(The block table has places for 64 positions: a rotary table of 63 is too short, unless the plan is made for no more.)"""
    refused(pkg.load_library().dmtd_paged_attention_shared(C.byref(cache()), C.byref(plan()), *dict(ATTENTION, **args).values(), None), word)


def test_small_memory_and_null_structs():
    lib, c = pkg.load_library(), cache()
    need, room = lib.dmtd_shared_plan_bytes(C.byref(c), 2), lib.dmtd_shared_workspace_bytes(C.byref(c))
    assert need > 0 and need % 256 == 0 and room > 0
    for p, word in ((plan(plan_bytes=need - 1), "plan's memory"), (plan(workspace_bytes=room - 1), "workspace")):
        refused(lib.dmtd_shared_plan_build(C.byref(c), C.byref(p), *BUILD.values(), None), word, pkg.DMTD_ECAPACITY)
        refused(lib.dmtd_paged_attention_shared(C.byref(c), C.byref(p), *ATTENTION.values(), None), word, pkg.DMTD_ECAPACITY)
    assert lib.dmtd_shared_plan_bytes(C.byref(c), 0) == lib.dmtd_shared_plan_bytes(C.byref(c), 8193) == lib.dmtd_shared_plan_bytes(None, 2) == lib.dmtd_shared_workspace_bytes(None) == 0
    refused(lib.dmtd_shared_plan_build(C.byref(c), None, *BUILD.values(), None), "null")
    refused(lib.dmtd_shared_plan_build(None, C.byref(plan()), *BUILD.values(), None), "null")
    refused(lib.dmtd_paged_attention_shared(C.byref(c), None, *ATTENTION.values(), None), "null")
    refused(lib.dmtd_paged_attention_shared(None, C.byref(plan()), *ATTENTION.values(), None), "null")


def ceil(a, b):
    return -(-a // b)


def floor_log2(v):
    return v.bit_length() - 1


@pytest.mark.parametrize("seed", range(40))
def test_the_memory_holds_every_plan(seed):
    """Items and units of partial results of random steps, by the plan's rules, against what the calls' sizes have room for."""
    import random
    rng = random.Random(seed)
    for _ in range(25):
        nkv, gq, f32 = rng.choice([1, 2, 3, 8, 16, 128]), rng.choice([1, 2, 4, 5, 7, 16]), rng.random() < 0.3
        page, n_req, n_groups = rng.choice([16, 32, 256]), rng.choice([1, 2, 5, 40, 300]), rng.choice([1, 2, 7, 40])
        few, tall = 16 // gq, 128 // gq
        slots = [1 << floor_log2(max(1024 // nkv, 1)), 1 << floor_log2(max(256 // nkv, 1))]
        rows = [rng.choice([0, 1, 1, 1, 2, 3, rng.randint(0, 400)]) for _ in range(n_req)]
        room = sum(rows) + rng.choice([0, 0, 3, 100]) or 1
        pages = [rng.choice([0, 1, rng.randint(1, 600)]) for _ in range(n_groups)]
        group, start = [rng.randint(-1, n_groups) for _ in range(n_req)], [rng.choice([0, rng.randint(0, 20000)]) for _ in range(n_req)]
        members = {g: [i for i in range(n_req) if group[i] == g and rows[i] and 0 < pages[g] * page <= start[i]] for g in range(n_groups)}
        entries, front = [], [0] * n_req
        for g, m in members.items():
            if len(m) > 1:
                entries.append((sum(rows[i] for i in m), pages[g] * page, True))
                for i in m:
                    front[i] = pages[g] * page
        entries += [(r, s + r - f, f > 0) for r, s, f in zip(rows, start, front) if r]
        kind = [not f32 and n * gq > 32 for n, _, _ in entries]
        per = [ceil(sum(ceil(e[0], tall if k else few) * e[1] for e, t in zip(entries, kind) if t == k), slots[k]) for k in (0, 1)]
        if per[1] >= 1536:
            in_all, tiles = sum(ceil(e[0], tall) * e[1] for e, t in zip(entries, kind) if t), sum(ceil(e[0], tall) for e, t in zip(entries, kind) if t)
            per[1] = ceil(in_all, 2 * slots[1] - (tiles if tiles < slots[1] else 0))
        keys = [max((64 if f32 else 128, 256)[k], ceil(per[k], 64) * 64) for k in (0, 1)]
        items = sum(ceil(n, tall if t else few) * ceil(length, keys[t]) for (n, length, _), t in zip(entries, kind))
        units = sum(n * ceil(length, keys[t]) for (n, length, apart), t in zip(entries, kind) if apart or ceil(length, keys[t]) > 1)
        c = cache(page_size=page, n_req=n_req, max_pages=2000, n_q_heads=nkv * gq, n_kv_heads=nkv, dtype=0 if f32 else 1, max_rows=room)
        lib = pkg.load_library()
        # behind a header of 64 bytes: 32 an item; a place and two records a row, 40; nine numbers a request and one more, seven a group
        assert 64 + 32 * items + 40 * room + 4 * (9 * n_req + 1 + 7 * n_groups) <= lib.dmtd_shared_plan_bytes(C.byref(c), n_groups)
        assert units * (nkv * gq * 64 + ceil(2 * nkv * gq, 4) * 4) * 4 <= lib.dmtd_shared_workspace_bytes(C.byref(c))


@pytest.mark.parametrize("args, word", [(dict(shared=P + 2), "aligned"), (dict(start=None), "null"), (dict(max_rows=0), "max_rows")])
def test_page_tables_with_shared_pages_refuses(args, word):
    a = dict(start=P, rows=P, shared=P, max_rows=8, cu=P, pos=P, slots=P, status=P)
    a.update(args)
    refused(pkg.load_library().dmtd_page_tables_shared(C.byref(pool()), *a.values(), None), word)
    assert set(TABLES) < set(a)
