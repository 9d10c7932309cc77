"""Attention over 8-bit caches keeps 16 bits of its probabilities, as that over bf16 caches does.

Scores are within a few hundredths of each other (queries of 2^-8) and values come in pairs v, -v, so that a result is what the probabilities of the pairs differ by, about 2^-8 of a value.
The tolerance is that of paged_util for queries and probabilities in two bf16 parts each: 2^-15 of sum p |v| and the output's own rounding, which is small where the output is.  Probabilities in
one part, each off by up to 2^-9 of itself, are up to 2^-9 of sum p |v| off, and 2^-12 root mean square at 16 keys."""
import pytest
import torch

from test_gpu_paged import H1, H4, H7, H8, H16, Setup
from test_gpu_paged8 import E8, Setup8
from test_gpu_paged_shared import attend, shared_setup

pytestmark = pytest.mark.gpu
SHORT = dict(norm=False, rope=False, spread=2.0 ** -8)


def cancel(s):
    """Every odd position's value is the one before it, negated (cached tokens and prefixes are even in number)."""
    odd = s.v[:, :, 1::2]
    s.v[:, :, 1::2] = torch.where(torch.isnan(odd), odd, -s.v[:, :, 0::2])
    # the newest tokens' values and keys are made small: a row sees some pairs' first value without the second
    for i, r in enumerate(s.rows):
        for p in range(s.start[i], s.start[i] + r):
            for t in (s.v, s.k):
                t[s.table[i][p // s.page], :, p % s.page] *= 2.0 ** -8
    s.store()
    return s


def check(s, got):
    ref, tol = Setup.reference(s)
    assert ref.abs().max() < 2.0 ** -4                # it cancels
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.numel(), ((got.double() - ref).abs() / tol).max().item())


@pytest.mark.parametrize("heads, page, start, rows", [
    (H8, 16, [14], [1]), (H4, 32, [30, 6, 200], [1, 1, 1]), (H16, 64, [1022], [1]), (H7, 16, [32, 60], [1, 3]), (H8, 16, [1998] * 8, [1] * 8),      # few rows
    (H8, 64, [200], [130]), (H4, 16, [0, 500], [65, 1]), (H1, 16, [30], [201]), (H7, 256, [130, 2], [75, 41]),                                   # many
])
def test_values_that_cancel(heads, page, start, rows):
    s = cancel(Setup8(heads, page, start, rows, seed=sum(start), **SHORT))
    check(s, s.attend())


@pytest.mark.parametrize("heads, page, pages, own, rows", [(H8, 16, 3, [14, 0, 200], [1, 1, 2]), (H4, 32, 20, [40, 6, 0, 100], [1, 3, 1, 2]), (H16, 16, 9, [10] * 12, [1] * 12), (H8, 64, 5, [20, 0], [90, 3])])
def test_values_that_cancel_behind_a_shared_prefix(heads, page, pages, own, rows):
    s = cancel(shared_setup(heads, E8, page, [pages], [0] * len(own), own, rows, seed=len(own), **SHORT))
    check(s, attend(s))
