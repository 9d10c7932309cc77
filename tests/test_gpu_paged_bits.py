"""The shared call without groups computes, bit for bit, what the unshared one does, where both take the same keys in the same order: requests of many rows over one range of keys, and
8-bit and fp32 requests of few rows over one group of 16 keys.  Which products of the queries' norm and rotation are rounded is written out for few rows; for many it is the
compiler's choice, and a build whose instantiations part shows here."""
import pytest
import torch

from test_gpu_paged import BF, F32, H1, H4, H7, H8, H16
from test_gpu_paged8 import E8
from test_gpu_paged_shared import attend, shared_setup

pytestmark = pytest.mark.gpu


def both(heads, dtype, page, start, rows, **kw):
    s = shared_setup(heads, dtype, page, [1], [-1] * len(start), start, rows, **kw)
    c = s.cache()
    a, b = s.attend(c), attend(s, c)
    s.check(a)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, E8])
@pytest.mark.parametrize("norm, rope", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("heads, page, start, rows", [(H8, 16, [100, 0], [90, 60]), (H4, 64, [0], [256]), (H7, 32, [150, 3], [40, 30]), (H1, 16, [31], [200]), (H16, 128, [201, 0], [55, 20])])
def test_many_rows(heads, dtype, page, start, rows, norm, rope):
    both(heads, dtype, page, start, rows, seed=sum(rows), norm=norm, rope=rope)


@pytest.mark.parametrize("dtype", [E8, F32])
@pytest.mark.parametrize("norm, rope", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("heads, page, start, rows", [(H8, 16, [0, 10, 3], [1, 3, 4]), (H4, 64, [5, 0], [8, 1]), (H7, 32, [9], [2]), (H1, 16, [0], [16]), (H16, 128, [14, 2], [1, 2])])
def test_few_rows(heads, dtype, page, start, rows, norm, rope):
    both(heads, dtype, page, start, rows, seed=sum(rows), norm=norm, rope=rope)
