"""Cross attention at the edges of its number range; bounds as in test_gpu_attend.py."""
import math

import pytest
import torch

from test_gpu_attend import TYPES, call, close, plain, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("lq,lk", [([3], [40]), ([3, 70], [40, 20]), ([130, 2], [300, 7]), ([1], [5000])])
@pytest.mark.parametrize("d", [30, 64, 128, 256])
def test_rows_of_infinitely_low_scores(d, lq, lk, dtype):
    """All scores of the first tree are -infinity, by infinite keys: zeros for its outputs and for every gradient, whatever its values hold; the other
    tree is as if alone."""
    s = tensors(31, TYPES[dtype], lq, lk, 2, 1, d)
    clean = call(s)
    nq, nk = lq[0], lk[0]
    s["q"][:nq] = 0
    s["q"][:nq, :, 0] = -1
    s["k"][:nk] = 0
    s["k"][:nk, :, 0] = math.inf
    for junk in (1.0, math.inf, -math.inf):
        s["v"][:nk] = junk
        got = call(s)
        assert (got["lse"][:nq] == -math.inf).all()
        for n in ("o", "d_q"):
            assert (got[n][:nq] == 0).all(), (n, junk)
            assert torch.equal(got[n][nq:], clean[n][nq:]), (n, junk)
        for n in ("d_k", "d_v"):
            assert (got[n][:nk] == 0).all(), (n, junk)
            assert torch.equal(got[n][nk:], clean[n][nk:]), (n, junk)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("lq,lk", [([3], [40]), ([37], [150]), ([9, 140], [300, 7])])
@pytest.mark.parametrize("d", [30, 64, 128, 256])
def test_a_key_at_minus_infinity_gets_no_gradient(d, lq, lk, dtype):
    """A node that every query of its tree scores -infinity: probabilities of zero, zero gradients of its key and value.  (d_q is 0 times that key: NaN.)"""
    s = tensors(32, TYPES[dtype], lq, lk, 2, 1, d)
    s["q"][:, :, 0] = s["q"][:, :, 0].abs() + 0.5
    s["k"][7, 0, 0] = -math.inf
    got = call(s)
    mask = torch.ones(sum(lk), dtype=torch.uint8, device="cuda")
    mask[7] = 0
    want, err = plain(dict(s, kv_mask=mask, k=s["k"].nan_to_num(neginf=0.0)))
    for n in ("o", "lse", "d_k", "d_v"):
        assert got[n].isfinite().all(), n
    assert (got["d_k"][7] == 0).all() and (got["d_v"][7] == 0).all()
    close(got, want, err, ["o", "lse", "d_k", "d_v"])
