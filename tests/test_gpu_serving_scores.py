"""Scores that are infinite: what the quotient of the definition has is what every attention kernel answers.

A score of +inf makes its row NaN (inf - inf in the exponent), wherever in a tile of the cache its token lies.  A row that sees
tokens, all with scores of -inf, is NaN too (0 / 0): only a row that sees no token at all is 0."""
import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests.test_gpu_serving import BF16, F32, Batch, ok

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


@pytest.mark.parametrize("kind,dtype,fresh", KINDS)
@pytest.mark.parametrize("lengths", [[1], [130, 1, 64], [1500]])
def test_minus_infinity_only(kind, dtype, fresh, lengths):
    b = batch(kind, dtype, fresh, lengths, seed=1)
    kept = b.k.clone()
    b.k[..., 0] = -INF                                   # every score
    with np.errstate(invalid="ignore"):
        out = b.check(max_q=fresh, kernel=kind)
        assert torch.isnan(out).all()
        assert torch.isnan(b.check(max_q=fresh, window=1, kernel=kind)).all()
        b.k.copy_(kept)
        for i, n in enumerate(lengths):                  # the last token alone: rows that see nothing else
            b.k[place(b, i, n - 1)][..., 0] = -INF
        out = b.check(max_q=fresh, kernel=kind)
        ends = np.cumsum(b.fresh) - 1
        assert all(bool(torch.isnan(out[e]).all()) == (n == 1) for e, n in zip(ends, lengths))
        out = b.check(max_q=fresh, window=1, kernel=kind)
        assert all(bool(torch.isnan(out[e]).all()) for e in ends)
    b.table.fill_(-1)                                    # and a row that sees no token is 0
    assert (b.check(max_q=fresh, kernel=kind) == 0).all()


@pytest.mark.parametrize("kind,dtype,fresh", KINDS)
def test_minus_infinity_in_part_of_the_cache(kind, dtype, fresh):
    """Whole tiles and whole parts of -inf beside finite scores: weights of 0."""
    for lo, hi in ((0, 1400), (0, 64), (640, 1500), (64, 1499)):
        b = batch(kind, dtype, fresh, [1500], seed=2)
        for token in range(lo, hi):
            b.k[place(b, 0, token)][..., 0] = -INF
        out = torch.full(b.q.shape, 7.0, dtype=F32, device="cuda")
        b.launch(b.code(out, scale=0.125, max_q=fresh), out)
        ok()
        assert dvm.last_attention_kernel() == kind
        assert torch.isfinite(out).all()
        with np.errstate(invalid="ignore"):
            # the bound's size of a score is infinite where a hidden element is: finite stand-ins that weigh nothing
            from tests.serving_oracle import attention, attention_bound, f64
            k = f64(b.k)
            gone = np.isneginf(k[..., 0])
            k[gone] = 0
            k[gone, 0] = -1e6
            want, mag, _, _, seen = attention(f64(b.q), k, f64(b.v), b.table.cpu().numpy(), b.starts.cpu().numpy(), b.lengths, 0.125, 0, 0)
            k[gone] = 0
            size = attention(f64(b.q), k, f64(b.v), b.table.cpu().numpy(), b.starts.cpu().numpy(), b.lengths, 0.125, 0, 0)[2]
        tol = attention_bound(want, mag, size, seen, 64, F32, dtype == BF16)
        assert (np.abs(f64(out) - want) <= tol).all()
