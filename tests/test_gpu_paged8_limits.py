"""Where 8-bit rows end: from 248 x 2^120 on, where an e4m3 code rounds to 2^128, values come back infinite; below, finite ones come back finite."""
import pytest
import torch

import paged8_util as p8
from test_gpu_paged import DEV, ints
from test_gpu_paged8 import Setup8

pytestmark = pytest.mark.gpu
TOP = 2.0 ** 120


@pytest.mark.parametrize("hd", [64, 128])
def test_the_largest_magnitudes(hd):
    tops = [1e38, 448.0 * 2.0 ** 119, 449.0 * 2.0 ** 119, 232.0 * TOP, 247.99 * TOP, 248.0 * TOP, 255.0 * TOP, 3.4028234663852886e38]
    rows = torch.stack([torch.linspace(-1, 1, hd, dtype=torch.float64).mul(m) for m in tops]).float()
    n = len(tops)
    s = Setup8((1, 1, hd), 16, [0], [n], norm=False, rope=False)
    s.qkv[:n, :hd], s.qkv[:n, hd:2 * hd], s.qkv[:n, 2 * hd:] = 0.0, rows, -rows
    c = s.cache()
    c.append(s.qkv.to(DEV), *s.maps())
    k, v = [t[:, 0].cpu().double() for t in c.read(ints(s.slots, torch.int64))]
    _, e, want = p8.stored(rows.double())
    assert e.tolist() == [245, 246] + [247] * 6
    beyond = rows.double().abs() >= 248.0 * TOP
    assert beyond.any(-1).tolist() == [m >= 248.0 * TOP for m in tops]
    for got, sign in ((k, 1), (v, -1)):
        assert torch.equal(torch.isinf(got), beyond) and not torch.isnan(got).any()
        assert torch.equal(got[~beyond], sign * want[~beyond])
