"""The 8-bit paged cache - append, read, attention - against plain 64-bit forms (paged_util, paged8_util), one by one and together."""
import numpy as np
import pytest
import torch

import paged8_util as p8
import paged_util as pu
import paper_2510_11958_amd as pkg
from test_gpu_paged import ATTENTION, BF, DEV, F32, H1, H4, H6, H7, H8, H16, Maps, Setup, ints

pytestmark = pytest.mark.gpu
E8 = torch.float8_e4m3fn


class Setup8(Setup):
    """Setup's keys and values as codes and scales; whatever no token lies in has codes and scales of all kinds, NaN among them."""

    def __init__(self, *args, **kw):
        super().__init__(args[0], BF, *args[1:], **kw)
        gen = torch.Generator().manual_seed(99)
        self.store(gen)

    def store(self, gen=None):
        for name in ("k", "v"):
            x = getattr(self, name)
            b, e, v = p8.stored(x.double())
            empty = torch.isnan(x).all(-1)
            if gen is not None:
                b[empty] = torch.randint(0, 256, b[empty].shape, generator=gen).to(torch.uint8)
                b[empty, 0] = 0x7F
                e[empty] = torch.randint(0, 256, e[empty].shape, generator=gen).to(torch.uint8)
            setattr(self, name, torch.where(empty[..., None], float("nan"), v.float()).to(BF))
            setattr(self, name + "b", b)
            setattr(self, name + "e", e)

    def cache(self, **kw):
        self.kd, self.vd = [t.view(E8) for t in kw.get("kv") or (self.kb.to(DEV), self.vb.to(DEV))]
        self.ksd, self.vsd = kw.get("scales") or (self.ke.to(DEV), self.ve.to(DEV))
        return pkg.PagedCache(self.kd, self.vd, ints(self.table), self.nq, self.room, k_scale=self.ksd, v_scale=self.vsd)

    def reference(self):
        return p8.attention(self.qkv, self.nq, self.k, self.v, self.table, self.page, self.start, self.rows, self.gain, self.rope, True)

    def maps(self):
        pad = self.room - self.total
        return ints(self.cu), ints(self.pos + [-1] * pad), ints(self.slots + [-1] * pad, torch.int64)


def at(t, slot, page):
    return t[slot // page, :, slot % page]


# ------------------------------------------------------------------------------------------ append

@pytest.mark.parametrize("heads, page, start, rows", [
    (H4, 16, [0], [1]), (H8, 32, [5], [3]), (H8, 16, [15, 16, 31], [1, 2, 17]), (H7, 256, [0, 300, 0], [0, 9, 1]), (H1, 64, [100, 0, 63, 64], [30, 70, 1, 0]), (H16, 128, [127, 0], [2, 40]),
])
@pytest.mark.parametrize("norm, rope", [(True, True), (False, False)])
def test_append(heads, page, start, rows, norm, rope):
    s = Setup8(heads, page, start, rows, seed=3, norm=norm, rope=rope)
    s.qkv[:s.total] *= torch.exp(2 * torch.randn(s.total, 1, generator=torch.Generator().manual_seed(1)))      # rows of all magnitudes
    c = s.cache()
    cu, pos, slots = s.maps()
    c.append(s.qkv.to(DEV), cu, pos, slots, k_norm=s.dev(s.gain), rope=s.dev(s.rope), eps=pu.EPS)
    slot = torch.tensor(s.slots)
    got = [t.cpu() for t in (s.kd.view(torch.uint8), s.vd.view(torch.uint8), s.ksd, s.vsd)]
    x = s.qkv[:s.total].double().view(s.total, -1, s.hd)
    # values are rounded as they are: bytes and scales are those of the plain form
    b, e, _ = p8.stored(x[:, s.nq + s.nkv:])
    assert torch.equal(at(got[1], slot, page), b) and torch.equal(at(got[3], slot, page), e)
    # keys: norm and rotation are off by hd + 10 roundings of the terms at most (as in the bf16 append); the scale is that of a maximum within that; the code is then within half a step
    want, mag = pu.normed_rotated(x[:, s.nq:s.nq + s.nkv], s.gain, s.rope, torch.tensor(s.pos))
    off = mag * (s.hd + 10) * pu.U32 if norm or rope else torch.zeros_like(mag)
    key_e = at(got[2], slot, page)
    lo, hi = p8.scale_bytes(torch.relu(want.abs() - off)), p8.scale_bytes(want.abs() + off)
    assert ((lo <= key_e) & (key_e <= hi)).all()
    key = p8.values(at(got[0], slot, page), key_e)
    assert ((key - want).abs() <= p8.half_step(want.abs() + off, key_e) + off).all()
    if not norm and not rope:
        b, e, _ = p8.stored(x[:, s.nq:s.nq + s.nkv])
        assert torch.equal(at(got[0], slot, page), b) and torch.equal(key_e, e)
    touched = torch.zeros(s.n_pages, page, dtype=torch.bool)
    touched[slot // page, slot % page] = True
    for g, was in zip(got, (s.kb, s.vb, s.ke, s.ve)):                  # every other place is as it was
        assert torch.equal(g.transpose(1, 2)[~touched], was.transpose(1, 2)[~touched])


@pytest.mark.parametrize("heads, norm, rope", [((8, 4, 128), True, True), ((8, 4, 64), True, True), ((8, 4, 128), True, False), ((8, 4, 64), False, True)])
def test_keys_are_rounded_from_more_than_32_bits(heads, norm, rope):
    """Half a million elements of keys: every code and scale is that of the 64-bit value.  Roundings of 32 bits, about 2^-23 of a key against codes 2^-4 to 2^-3 of it apart, would have about one of a
    million on the other side of a border; those of 64 bits are 2^-29 as many."""
    s = Setup8(heads, 32, [100, 0], [700, 400], seed=23, norm=norm, rope=rope)
    c = s.cache()
    cu, pos, slots = s.maps()
    for seed in range(3):
        s.qkv[:s.total] = torch.randn(s.total, s.qkv.shape[1], generator=torch.Generator().manual_seed(seed))
        c.append(s.qkv.to(DEV), cu, pos, slots, k_norm=s.dev(s.gain), rope=s.dev(s.rope), eps=pu.EPS)
        x = s.qkv[:s.total].double().view(s.total, -1, s.hd)
        want, _ = pu.normed_rotated(x[:, s.nq:s.nq + s.nkv], s.gain, s.rope, torch.tensor(s.pos))
        b, e, _ = p8.stored(want)
        slot = torch.tensor(s.slots)
        assert torch.equal(at(s.ksd.cpu(), slot, s.page), e)
        assert torch.equal(at(s.kd.view(torch.uint8).cpu(), slot, s.page), b)


def test_append_at_the_borders_of_codes_and_scales():
    """Rows around each power of two's limit, halves between codes, subnormal codes, zeros, the smallest and largest magnitudes, and values that are not finite."""
    hd, page = 64, 16
    border = []
    for most in [448.0, 448.0 * (1 + 2.0 ** -23), 448.0 * (1 - 2.0 ** -24), 0.0, 1e-45, 1e-38, 448.0 * 2.0 ** -111, 449.0 * 2.0 ** -111, 1e-30, 3e38, 3.4028234663852886e38, 1.0, 1.75, 1.7500001]:
        y = torch.linspace(-1, 1, hd, dtype=torch.float64) * most
        y[0] = most
        border.append(y)
    every = torch.arange(0x7F, dtype=torch.uint8).view(E8).double()
    halves = torch.cat([(every[1:] + every[:-1]) / 2, torch.zeros(2, dtype=torch.float64)]).view(2, hd)
    halves[:, -1] = 448.0
    odd = torch.randn(6, hd, dtype=torch.float64, generator=torch.Generator().manual_seed(2))
    odd[0, 5], odd[1, 0], odd[2, 63], odd[4, :] = float("nan"), float("inf"), -float("inf"), float("nan")
    odd[5, 1:] = float("inf")
    rows = torch.cat([torch.stack(border), halves, -halves, odd]).float()
    n = rows.shape[0]
    s = Setup8((1, 1, hd), page, [0], [n], norm=False, rope=False)
    s.qkv[:n, :hd], s.qkv[:n, hd:2 * hd], s.qkv[:n, 2 * hd:] = 0.0, rows, rows.flip(0)
    c = s.cache()
    c.append(s.qkv.to(DEV), *s.maps())
    slot = torch.tensor(s.slots)
    for codes, scales, x in ((s.kd, s.ksd, rows), (s.vd, s.vsd, rows.flip(0))):
        b, e, v = p8.stored(x.double())
        got, got_e = at(codes.view(torch.uint8).cpu(), slot, page)[:, 0], at(scales.cpu(), slot, page)[:, 0]
        assert torch.equal(got_e, e)
        nan = (b & 0x7F) == 0x7F
        assert torch.equal((got & 0x7F) == 0x7F, nan) and torch.equal(got[~nan], b[~nan])


def test_append_leaves_out_bad_places():
    s = Setup8(H4, 16, [3, 0], [4, 2])
    c, n = s.cache(), s.n_pages * 16
    pad = s.room - s.total
    slots = [n, -1, s.slots[2], -(1 << 40), 1 << 40, s.slots[5]]
    pos = [s.pos[0], s.pos[1], -1, s.pos[3], s.pos[4], s.width * 16]
    c.append(s.qkv.to(DEV), ints(s.cu), ints(pos + [0] * pad), ints(slots + [0] * pad, torch.int64), k_norm=s.dev(s.gain), rope=s.dev(s.rope))
    torch.cuda.synchronize()
    for got, was in ((s.kd.view(torch.uint8), s.kb), (s.vd.view(torch.uint8), s.vb), (s.ksd, s.ke), (s.vsd, s.ve)):
        assert torch.equal(got.cpu(), was)


# ------------------------------------------------------------------------------------------ read

def filled(heads, dtype, page, n_pages, apart=0, seed=0):
    """A pool with something everywhere, its handle, and its values as the wide type; apart: elements between pages."""
    nq, nkv, hd = heads
    gen = torch.Generator().manual_seed(seed)
    shape = (n_pages, nkv, page, hd)
    x = [torch.randn(shape, generator=gen) for _ in range(2)]
    table = ints([[0]])

    def spread(t, gap):
        size = t[0].numel() + gap
        out = torch.empty(size * n_pages, dtype=t.dtype, device=DEV).as_strided(t.shape, (size,) + t.stride()[1:])
        out.copy_(t.to(DEV))
        return out

    if dtype is not E8:
        wide = [t.to(dtype) for t in x]
        return pkg.PagedCache(spread(wide[0], apart), spread(wide[1], apart), table, nq, 4), wide
    st = [p8.stored(t.double()) for t in x]
    codes, scales = [spread(b, apart).view(E8) for b, _, _ in st], [spread(e, apart) for _, e, _ in st]
    return pkg.PagedCache(codes[0], codes[1], table, nq, 4, k_scale=scales[0], v_scale=scales[1]), [v.to(BF) for _, _, v in st]


@pytest.mark.parametrize("dtype", [E8, BF, F32])
@pytest.mark.parametrize("heads, page, n, apart", [(H4, 16, 1, 0), (H8, 16, 33, 0), (H7, 64, 100, 64), (H1, 256, 1000, 0), (H16, 32, 17, 16), (H6, 128, 5, 0)])
def test_read(heads, dtype, page, n, apart):
    c, (k, v) = filled(heads, dtype, page, 5, apart)
    rng = np.random.RandomState(n)
    slots = rng.randint(0, 5 * page, n)                                # any order, the same place more than once
    if n > 20:
        slots[[3, 9]] = slots[4]
    out = [torch.full((n, heads[1], heads[2]), 9.0, dtype=BF if dtype is E8 else dtype, device=DEV) for _ in range(2)]
    got = c.read(ints(slots, torch.int64), *out)
    assert got[0] is out[0] and got[1] is out[1]
    where = torch.tensor(slots)
    assert torch.equal(out[0].cpu(), at(k, where, page)) and torch.equal(out[1].cpu(), at(v, where, page))
    again = c.read(ints(slots, torch.int64))
    assert torch.equal(again[0], out[0]) and torch.equal(again[1], out[1])


@pytest.mark.parametrize("dtype", [E8, BF, F32])
def test_read_leaves_out_bad_places(dtype):
    c, (k, v) = filled(H8, dtype, 16, 3)
    slots = [5, -1, 48, 47, 1 << 40, -(1 << 40), 0]
    out = [torch.full((7, 2, 128), 9.0, dtype=c.dtype, device=DEV) for _ in range(2)]
    c.read(ints(slots, torch.int64), *out)
    for o, x in zip(out, (k, v)):
        for t, p in enumerate(slots):
            assert torch.equal(o[t].cpu(), x[p // 16, :, p % 16] if 0 <= p < 48 else torch.full((2, 128), 9.0, dtype=c.dtype))
    e = c.read(ints([], torch.int64))
    assert e[0].shape == e[1].shape == (0, 2, 128)


def test_read_of_every_code_and_scale():
    """256 codes under every scale byte: code x 2^(e - 127), rounded to bf16 where it is not one (below the least scale that append writes); NaN under 255."""
    page = 256
    b = torch.arange(256, dtype=torch.uint8).view(2, 128)
    kb = b[None, :, None].expand(1, 2, page, 128).contiguous()
    e = torch.arange(256, dtype=torch.uint8)[None, None].expand(1, 2, page).contiguous()
    c = pkg.PagedCache(kb.to(DEV).view(E8), kb.flip(-1).contiguous().to(DEV).view(E8), ints([[0]]), 2, 4, k_scale=e.to(DEV), v_scale=e.to(DEV))
    k, v = [t.cpu() for t in c.read(torch.arange(256, device=DEV))]
    want = p8.values(kb[0].transpose(0, 1).contiguous(), e[0].t().contiguous()).float().to(BF)
    for got, w in ((k, want), (v, want.flip(-1))):
        assert torch.equal(got.isnan(), w.isnan()) and torch.equal(got[~w.isnan()], w[~w.isnan()])


# ------------------------------------------------------------------------------------------ attention

@pytest.mark.parametrize("heads, page, start, rows", ATTENTION)
def test_attention(heads, page, start, rows):
    Setup8(heads, page, start, rows, seed=len(start) + sum(rows)).check()


@pytest.mark.parametrize("norm, rope", [(True, False), (False, True), (False, False)])
def test_attention_without_norm_or_rotation(norm, rope):
    Setup8(H8, 32, [70, 0, 200], [1, 40, 3], seed=5, norm=norm, rope=rope).check()


def test_ranges_longer_than_a_wave_keeps_page_numbers_for():
    Setup8((128, 128, 64), 16, [8999], [1], seed=21).check()


def test_large_scores():
    Setup8(H8, 16, [300, 40], [1, 90], seed=6, norm=False, spread=100.0).check()


def test_rows_of_all_magnitudes():
    """Keys and values of every magnitude from 1e-30 to 1e30 a row: the scales, not the codes, carry them (queries so short that scores stay within reach)."""
    s = Setup8(H8, 16, [90, 30], [1, 60], seed=14, norm=False, rope=False)
    gen = torch.Generator().manual_seed(4)
    s.v = (s.v.double() * 10 ** (60 * torch.rand(s.v.shape[:3], generator=gen, dtype=torch.float64)[..., None] - 30)).to(BF)
    s.k = (s.k.double() * 10 ** (6 * torch.rand(s.k.shape[:3], generator=gen, dtype=torch.float64)[..., None] - 5)).to(BF)
    s.store(gen)
    s.check()


@pytest.mark.parametrize("rows", [[1, 1], [3, 2], [90, 40]])
def test_pages_apart_and_wide_rows(rows):
    """Codes and scales of K and V interleaved in one allocation each, rows of qkv and of out wider than what they hold."""
    s = Setup8(H8, 32, [100, 7], rows, seed=8)
    both = torch.full((s.n_pages, 2) + s.kb.shape[1:], 0x7F, dtype=torch.uint8, device=DEV)
    scales = torch.full((s.n_pages, 3) + s.ke.shape[1:], 255, dtype=torch.uint8, device=DEV)
    both[:, 0], both[:, 1], scales[:, 0], scales[:, 1] = s.kb.to(DEV), s.vb.to(DEV), s.ke.to(DEV), s.ve.to(DEV)
    c = s.cache(kv=(both[:, 0], both[:, 1]), scales=(scales[:, 0], scales[:, 1]))
    wide = torch.full((s.room, s.qkv.shape[1] + 12), float("nan"), device=DEV)
    wide[:, :s.qkv.shape[1]] = s.qkv.to(DEV)
    out = torch.full((s.room, s.nq + 1, s.hd), 5.0, dtype=BF, device=DEV)
    c.attention(wide[:, :s.qkv.shape[1]], ints(s.start), ints(s.cu), out[:, :s.nq], q_norm=s.dev(s.gain), rope=s.dev(s.rope))
    assert (out[:, s.nq] == 5.0).all() and (out[s.total:] == 5.0).all()
    s.check(out[:s.total, :s.nq].cpu())
    c.append(wide[:, :s.qkv.shape[1]], *s.maps(), k_norm=s.dev(s.gain), rope=s.dev(s.rope))
    slot = torch.tensor(s.slots)
    b, e, _ = p8.stored(s.qkv[:s.total].double().view(s.total, -1, s.hd)[:, s.nq + s.nkv:])
    assert torch.equal(at(both[:, 1].cpu(), slot, 32), b) and torch.equal(at(scales[:, 1].cpu(), slot, 32), e)
    assert (scales[:, 2] == 255).all()


@pytest.mark.parametrize("start, rows", [([20], [5]), ([0, 100], [1, 3]), ([0], [90]), ([70, 30], [130, 1])])
@pytest.mark.parametrize("how", ["code", "scale"])
def test_later_values_that_are_nan(start, rows, how):
    """The newest token's value (and the one's in the middle of a chunk) is NaN, in one code or by its scale: the rows before it come out as if it were not, those that see it do not."""
    s = Setup8(H8, 16, start, rows, seed=9)
    ref, tol = s.reference()
    mid = rows[0] - 1 - rows[0] // 3
    for i, j in ((0, mid), (len(rows) - 1, rows[-1] - 1)):
        p = start[i] + j
        if how == "code":
            s.vb[s.table[i][p // 16], :, p % 16, 3] = 0xFF
        else:
            s.ve[s.table[i][p // 16], :, p % 16] = 255
    got = s.attend()
    for i in range(len(rows)):
        first = {0: mid}.get(i, rows[i]) if i == 0 else rows[i]
        if i == len(rows) - 1:
            first = min(first, rows[i] - 1)
        a, b = s.cu[i], s.cu[i] + first
        assert ((got[a:b].double() - ref[a:b]).abs() <= tol[a:b]).all()
        assert torch.isnan(got[b:s.cu[i + 1], :, 3]).all()


@pytest.mark.parametrize("rows", [[1, 1, 1], [4, 3, 2], [100, 70, 33]])
def test_missing_pages(rows):
    s = Setup8(H8, 16, [80, 40, 0], rows, seed=10)
    s.table[0][1], s.table[0][3] = -1, s.n_pages
    s.table[1][0] = 1 << 30
    s.table[2] = [-1] * s.width
    ref, tol = s.reference()
    assert (ref[s.cu[2]:] == 0).all()
    s.check()


def test_lengths_that_do_not_fit_are_left_out():
    s = Setup8(H8, 16, [30, 20, 50, 10], [2, 3, 40, 1], seed=11)
    c = s.cache()
    good = s.attend(c)
    s.check(good)
    limit = s.width * 16
    for start, cu, skipped in [([30, -1, 50, 10], s.cu, 1), ([30, limit - 2, 50, 10], s.cu, 1), ([30, 20, 50, 10], s.cu[:4] + [s.room + 1], 3)]:
        out = torch.full((s.room, s.nq, s.hd), 77.0, dtype=BF, device=DEV)
        c.attention(s.qkv.to(DEV), ints(start), ints(cu), out, q_norm=s.dev(s.gain), rope=s.dev(s.rope))
        out = out.cpu()
        for i in range(4):
            a, b = s.cu[i], s.cu[i + 1]
            assert (out[a:b] == 77.0).all() if i == skipped else torch.equal(out[a:b], good[a:b])


@pytest.mark.parametrize("rows", [[1, 1, 1], [100, 1, 2]])
def test_pages_beyond_32_bit_offsets(rows):
    """Pages of codes 2^28 bytes apart and their scales 2^28 too: those from number 8 on lie beyond 2^31, from 16 on beyond 2^32."""
    s = Setup8((4, 2, 64), 16, [100, 60, 130], rows, seed=12)
    gap = 1 << 28
    far = []
    for src in (s.kb, s.vb, s.ke, s.ve):
        flat = torch.empty((s.n_pages - 1) * gap + src[0].numel(), dtype=torch.uint8, device=DEV)
        t = flat.as_strided(src.shape, (gap,) + src.stride()[1:])
        t.copy_(src.to(DEV))
        far.append(t)
    assert s.n_pages > 17 and max(max(r) for r in s.table) >= 17
    c = s.cache(kv=tuple(far[:2]), scales=tuple(far[2:]))
    s.check(s.attend(c))
    slot = torch.tensor(s.slots, device=DEV)
    k, v = c.read(slot)
    assert torch.equal(v.cpu(), at(s.v, slot.cpu(), 16))
    c.append(s.qkv.to(DEV), *s.maps(), k_norm=s.dev(s.gain), rope=s.dev(s.rope))
    b, e, _ = p8.stored(s.qkv[:s.total].double().view(s.total, -1, 64)[:, 6:])
    assert torch.equal(at(far[1], slot, 16).cpu(), b) and torch.equal(at(far[3], slot, 16).cpu(), e)


def test_many_requests():
    rng = np.random.RandomState(3)
    for n in (65, 300):
        Setup8(H4, 16, rng.randint(0, 40, n).tolist(), rng.randint(0, 3, n).tolist(), seed=n).check()
    start, rows = rng.randint(0, 700, 90), rng.randint(0, 5, 90)
    start[[7, 50, 88]], rows[[7, 50, 88]] = [0, 900, 2100], [150, 77, 130]
    s = Setup8(H4, 32, start.tolist(), rows.tolist(), seed=23)
    s.check()
    assert torch.equal(s.attend(max_new=150), s.attend())


def test_same_bits_every_time_and_on_every_stream():
    s = Setup8(H8, 64, [3000, 10, 0, 500], [1, 90, 1, 5], seed=13)
    c = s.cache()
    first = s.attend(c)
    side = torch.cuda.Stream()
    for turn in range(6):
        with torch.cuda.stream(side if turn % 2 else torch.cuda.current_stream()):
            assert torch.equal(s.attend(c), first)
        torch.cuda.synchronize()


def test_layers_of_all_types_share_a_workspace():
    layers = [Setup8(H8, 32, [2000] + [300] * 60, [1] * 61, seed=33), Setup(H8, BF, 32, [2000] + [300] * 60, [1] * 61, seed=33), Setup(H8, F32, 32, [2000] + [300] * 60, [1] * 61, seed=33)]
    first = layers[0].cache()
    handles = [first] + [first.layer(s.k.to(DEV), s.v.to(DEV)) for s in layers[1:]] + [first.layer(first.k, first.v, k_scale=first.k_scale, v_scale=first.v_scale)]
    for _ in range(2):
        for s, c in zip(layers + layers[:1], handles):
            s.check(s.attend(c))


def test_the_handles_check_their_tensors():
    s = Setup8(H8, 32, [40], [3], seed=31)
    c = s.cache()
    table = c.block_table
    bad = [dict(k_scale=None), dict(v_scale=s.vsd.float()), dict(k_scale=s.ksd[:-1]), dict(v_scale=s.vsd.cpu()), dict(k_scale=s.ksd.transpose(1, 2).contiguous().transpose(1, 2)),
           dict(k_scale=torch.zeros(s.n_pages, 2, 64, dtype=torch.uint8, device=DEV)[:, :, :32])]
    for b in bad:
        with pytest.raises(ValueError):
            pkg.PagedCache(s.kd, s.vd, table, s.nq, s.room, **dict(dict(k_scale=s.ksd, v_scale=s.vsd), **b))
    with pytest.raises(ValueError):
        pkg.PagedCache(s.k.to(DEV), s.v.to(DEV), table, s.nq, s.room, k_scale=s.ksd, v_scale=s.vsd)
    with pytest.raises(ValueError):
        pkg.PagedCache(s.kd, s.k.to(DEV), table, s.nq, s.room, k_scale=s.ksd, v_scale=s.vsd)
    with pytest.raises(ValueError):
        pkg.PagedCache(s.kd.view(torch.uint8), s.vd.view(torch.uint8), table, s.nq, s.room, k_scale=s.ksd, v_scale=s.vsd)
    with pytest.raises(ValueError):
        c.attention(s.qkv.to(DEV), ints(s.start), ints(s.cu), torch.zeros(s.room, 8, 128, dtype=E8, device=DEV))
    slots = ints([1, 2], torch.int64)
    wide = torch.zeros(2, 2, 128, dtype=BF, device=DEV)
    for a in ((slots.int(),), (slots.cpu(),), (slots[None],), (ints([1, 2, 3, 4], torch.int64)[::2],), (slots, wide.float()), (slots, wide[:1]), (slots, wide, wide[:, :1]), (slots, wide.cpu())):
        with pytest.raises(ValueError):
            c.read(*a)


# ------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("heads, page", [(H8, 16), (H4, 32), (H7, 64)])
def test_the_operators_together(heads, page, graph):
    """A small server over an 8-bit pool: requests arrive, bring a prompt in chunks, then tokens one by one, and end.  What append stored is read back and held to the plain form; every
    step's outputs are held to the plain attention over what has been read."""
    nq, nkv, hd = heads
    n_pages, n_req, max_pages, room = 400 * 16 // page, 6, 320 // page, 256
    rng, gen = np.random.RandomState(4), torch.Generator().manual_seed(4)
    tables = pkg.PageTables.empty(n_pages, page, n_req, max_pages, DEV)
    codes = [torch.full((n_pages, nkv, page, hd), 0x7F, dtype=torch.uint8, device=DEV).view(E8) for _ in range(2)]
    scales = [torch.full((n_pages, nkv, page), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
    cache = pkg.PagedCache(codes[0], codes[1], tables.block_table, nq, room, k_scale=scales[0], v_scale=scales[1])
    gain_q, gain_k = [(1 + 0.2 * torch.randn(hd, generator=gen)).to(BF) for _ in range(2)]
    rope = pu.rope_table(max_pages * page, hd)
    start_d, rows_d, m = ints([0] * n_req), ints([0] * n_req), Maps(n_req, room)
    qkv_d, out_d = torch.zeros(room, (nq + 2 * nkv) * hd, device=DEV), torch.zeros(room, nq, hd, dtype=BF, device=DEV)
    back = [torch.zeros(room, nkv, hd, dtype=BF, device=DEV) for _ in range(2)]
    gq, gk, rp = gain_q.to(DEV), gain_k.to(DEV), rope.to(DEV)

    def step():
        tables.build(start_d, rows_d, *m.all())
        cache.append(qkv_d, m.cu, m.pos, m.slots, k_norm=gk, rope=rp)
        cache.read(m.slots, *back)
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
    for turn in range(12):
        rows = []
        for i in range(n_req):
            if cached[i] and rng.rand() < 0.15:
                cached[i], keys[i], values[i] = 0, None, None
                rows.append(0)
            elif cached[i] == 0:
                rows.append(int(rng.choice([1, 20, 70, 130])) if rng.rand() < 0.7 else 0)
            else:
                rows.append(int(rng.randint(0, 4)))
            if cached[i] + rows[i] > max_pages * page or sum(rows) > room:
                rows[i] = 0
        total = sum(rows)
        qkv = torch.randn(room, qkv_d.shape[1], generator=gen)
        qkv_d.copy_(qkv)
        out_d.fill_(3.0)
        m.slots.fill_(-1)                                             # rows behind the last one: nothing to read
        start_d.copy_(ints(cached))
        rows_d.copy_(ints(rows))
        g.replay() if g else step()
        torch.cuda.synchronize()
        assert m.status.tolist() == [0, 0] and m.cu[-1].item() == total
        got, new_k, new_v = out_d.cpu(), back[0][:total].cpu(), back[1][:total].cpu()
        a = 0
        for i, r in enumerate(rows):
            if r == 0:
                continue
            x = qkv[a:a + r].view(r, -1, hd)
            pos = torch.arange(cached[i], cached[i] + r)
            want, mag = pu.normed_rotated(x[:, nq:nq + nkv].double(), gain_k, rope, pos)
            off = mag * (hd + 10) * pu.U32
            assert ((new_k[a:a + r].double() - want).abs() <= p8.half_step(want.abs() + off, p8.scale_bytes(want.abs() + off)) + off).all()
            assert torch.equal(new_v[a:a + r].double(), p8.stored(x[:, nq + nkv:])[2])
            keys[i] = new_k[a:a + r] if keys[i] is None else torch.cat([keys[i], new_k[a:a + r]])
            values[i] = new_v[a:a + r] if values[i] is None else torch.cat([values[i], new_v[a:a + r]])
            n = keys[i].shape[0]
            ref, tol = p8.attention(x[:, :nq].reshape(r, -1), nq, keys[i].transpose(0, 1)[None], values[i].transpose(0, 1)[None], [[0]], n, [cached[i]], [r], gain_q, rope, True)
            assert ((got[a:a + r].double() - ref).abs() <= tol).all()
            cached[i] += r
            a += r
        assert (got[total:] == 3.0).all()
