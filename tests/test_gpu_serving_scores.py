"""Scores that are infinite: what the quotient of the definition has is what every attention kernel answers.

A score of +inf makes its row NaN (inf - inf in the exponent), wherever in a tile of the cache its token lies."""
import numpy as np
import pytest
import torch

from tests.test_gpu_serving import BF16, F32, Batch

pytestmark = pytest.mark.gpu

INF = float("inf")
KINDS = [("prompt", BF16, 66), ("prompt", BF16, 2), ("single", BF16, 1), ("plain", F32, 66), ("plain", F32, 1)]


def batch(kind, dtype, fresh, lengths, dim=64, page=16, hq=2, hk=1, seed=0):
    """Queries whose first element is at least 1, so that an infinite first element of a key decides its score."""
    b = Batch(lengths, [min(fresh, n) for n in lengths], hq, hk, dim, page, dtype=dtype, seed=seed)
    b.q[..., 0] = b.q[..., 0].abs() + 1
    return b


def place(b, request, token):
    return int(b.table[request, token // b.page]), token % b.page


@pytest.mark.parametrize("kind,dtype,fresh", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
def test_plus_infinity_at_every_place_of_a_tile(kind, dtype, fresh, dim):
    b = batch(kind, dtype, fresh, [131], dim=dim)
    for token in range(64, 131):                         # every place of a tile that all rows see, or that is cut by the mask
        at = place(b, 0, token)
        kept = b.k[at].clone()
        b.k[at][..., 0] = INF
        with np.errstate(invalid="ignore"):
            out = b.check(max_q=fresh, kernel=kind)
        assert torch.isnan(out[max(0, token - 131 + out.shape[0]):]).all()
        b.k[at] = kept


@pytest.mark.parametrize("kind,dtype,fresh", KINDS)
def test_plus_infinity_far_from_the_end(kind, dtype, fresh):
    """The rows' maximum is infinite from an early tile on, or becomes it late, in one of several parts of the cache."""
    b = batch(kind, dtype, fresh, [1500, 40])
    for token in (3, 700, 701, 1400):
        at = place(b, 0, token)
        kept = b.k[at].clone()
        b.k[at][..., 0] = INF
        with np.errstate(invalid="ignore"):
            out = b.check(max_q=fresh, kernel=kind)
        first = min(fresh, 1500)
        assert torch.isnan(out[:first]).all() and torch.isfinite(out[first:]).all()
        b.k[at] = kept
