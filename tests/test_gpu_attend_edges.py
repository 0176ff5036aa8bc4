"""Cross attention at the edges of its number range: infinite inputs, probabilities far below the largest, gradients given what tl_attend stored.

stored() has what tl_attend_backward returns for the o and lse that it is given, in 64 bits, so that the rounding of o is an input and no error.
With u = 2^-24 and h = half a step of the operands' type:
  probability 2^x of a sum of D products, two roundings of the scale, lse in base 2, the fp16 forms' shift by 2^14 and the difference:
              relative |ds| + (4 |s| + 4 |lse| + 24) u  with  |ds| <= (D + 4) u * scale * sum |q||k|; 0 below 2^-126, as are operands
  as operand  16 bits in one term: h; in two terms: h^2, of what the first left; fp16, shifted by 2^14, below its normal range 2^-25 2^-14
  score gradient  P (dP - delta): that of P, (D + 4) u of both sums' absolute values; two terms: h^2.  fp16: a row of d_o is brought to a length of
              2^9 .. 2^10, and where a score gradient passes 2^15 it is brought to that: 2^-25 2^-9 of the larger one below the normal range
  sums        (2 n + 8) u of the products' absolute values (two terms are two products); rounded once to the type.
"""
import math

import pytest
import torch

from paper_1809_00832_amd import binding
from test_gpu_attend import TYPES, U, call, close, half_step, plain, tensors, where

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


def stored(s, o, lse, p_terms):
    """d_q, d_k, d_v from o and lse, and a bound of the error of each.  p_terms: 16-bit terms of a probability in d_v's product."""
    q, k, v, g, o = (x.double() for x in (s["q"], s["k"], s["v"], s["d_o"], o))
    lse = lse.double()
    dtype, scale = s["q"].dtype, s["scale"]
    G, D = q.shape[1] // k.shape[1], q.shape[2]
    h = half_step(dtype) if dtype != torch.float32 else 0.0
    f16 = dtype == torch.float16
    out = {"d_q": torch.zeros_like(q), "d_k": torch.zeros_like(k), "d_v": torch.zeros_like(v)}
    err = {n: torch.zeros_like(x) for n, x in out.items()}
    a = b = 0
    for nq, nk in zip(s["lq"], s["lk"]):
        rows, cols = slice(a, a + nq), slice(b, b + nk)
        a, b = a + nq, b + nk
        for j in range(q.shape[1]):
            Q, K, V, dO, O, L = q[rows, j], k[cols, j // G], v[cols, j // G], g[rows, j], o[rows, j], lse[rows, j, None]
            S = Q @ K.t() * scale
            P = torch.exp(S - L)
            rel = (D + 4) * U * scale * (Q.abs() @ K.abs().t()) + (4 * S.abs() + 4 * L.abs() + 24) * U
            gap = dO @ V.t() - (dO * O).sum(1, keepdim=True)
            dS = P * gap
            e_dS = rel * dS.abs() + P * (1 + rel) * ((D + 4) * U * (dO.abs() @ V.abs().t() + (dO.abs() * O.abs()).sum(1, keepdim=True)) + 2 * U * gap.abs())
            e_dS = e_dS + h * h * (dS.abs() + e_dS) + 2.0 ** -126 * gap.abs() + 2.0 ** -125
            low_q = low_k = 0.0
            if f16:
                size, top = dO.norm(dim=1, keepdim=True), dS.abs()
                low_q = 2.0 ** -34 * torch.maximum(size, top.amax(1, keepdim=True))
                low_k = 2.0 ** -34 * torch.maximum(size.amax(), top.amax(0, keepdim=True))
            m = nq * G
            e_P = (rel + h ** p_terms) * P + (2.0 ** -39 if f16 else 2.0 ** -125)
            dq, dk, dv = scale * dS @ K, scale * dS.t() @ Q, P.t() @ dO
            e_q = scale * ((e_dS + low_q) @ K.abs() + (2 * nk + 8) * U * (dS.abs() @ K.abs()))
            out["d_q"][rows, j], err["d_q"][rows, j] = dq, e_q
            out["d_k"][cols, j // G] += dk
            out["d_v"][cols, j // G] += dv
            err["d_k"][cols, j // G] += scale * ((e_dS + low_k).t() @ Q.abs() + (2 * m + 8) * U * (dS.abs().t() @ Q.abs()))
            err["d_v"][cols, j // G] += e_P.t() @ dO.abs() + (2 * m + 8) * U * (P.t() @ dO.abs())
    for n in out:
        err[n] = err[n] + half_step(dtype) * (out[n].abs() + err[n]) + (2.0 ** -25 if f16 else 1e-36)
    return out, err


def gradients(s):
    o, lse = binding.tl_attend(s["q"], s["k"], s["v"], with_lse=True, **where(s))
    return o, lse, binding.tl_attend_backward(s["q"], s["k"], s["v"], o, lse, s["d_o"], **where(s))


@pytest.mark.parametrize("lq", [[1], [40], [300]])
def test_fp16_outputs_of_many_small_probabilities(lq):
    """One node far ahead of the others, whose probabilities are some 2^-22 each: unscaled they would be four or five of fp16's smallest steps.  The leading
    node's value is zero, so that the output is made of the others alone (in one tile with it: a list this short is not divided)."""
    d, n = 64, 250
    s = tensors(33, torch.float16, lq, [n], 1, 1, d)
    s["q"][:], s["k"][:] = 0, 0
    s["q"][:, 0, 0] = 8
    s["k"][17, 0, 0] = 15.13                                  # times 8 / sqrt(64): the score, beside zeros
    s["v"][:] = s["v"].abs() + 1
    s["v"][17] = 0
    got, _ = binding.tl_attend(s["q"], s["k"], s["v"], with_lse=True, **where(s))
    Q, K, V = (s[name].double()[:, 0] for name in "qkv")
    P = torch.softmax(Q @ K.t() * s["scale"], 1)
    O = P @ V
    h = half_step(torch.float16)
    e = (2 * (d + 4) * U * 15.2 + (8 * 15.2 + n + 24) * U + h) * O + 2.0 ** -39 * V.sum(0)
    e = e + h * (O + e)
    assert ((got[:, 0].double() - O).abs() <= e).all(), float(((got[:, 0].double() - O).abs() / e).max())


@pytest.mark.parametrize("lq,lk,terms", [([600], [20000], 2), ([900, 31], [90, 120], 2), ([64], [16384], 2)])
@pytest.mark.parametrize("size", [1.0, 512.0])
def test_fp16_value_gradients_of_small_probabilities(lq, lk, terms, size):
    """Probabilities far below fp16's normal range, with upstream gradients of a scaled loss: d_v of every node."""
    s = tensors(34, torch.float16, lq, lk, 1, 1, 64, spread=1.0)
    s["q"] *= 2
    s["d_o"] *= size
    o, lse, got = gradients(s)
    ref, err = stored(s, o, lse, terms)
    fits = {n: ref[n].abs() < 6e4 for n in ref}
    for n in ref:
        bad = fits[n] & ~((got[n].double() - ref[n]).abs() <= err[n])
        assert fits[n].float().mean() > 0.99 and not bad.any(), (n, int(bad.sum()))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads,kv_heads,d,lq,lk,p_terms", [(4, 2, 64, [33, 60, 5], [54, 99, 9], 2), (2, 1, 128, [700, 40], [900, 600], 1),
                                                            (1, 1, 256, [100, 9], [300, 40], 2), (6, 3, 30, [200, 90], [100, 90], 2)])
def test_gradients_from_what_was_stored(heads, kv_heads, d, lq, lk, p_terms, dtype):
    """Score gradients in one term of 16 bits, or such probabilities where two are promised, would pass these bounds by far."""
    s = tensors(35, TYPES[dtype], lq, lk, heads, kv_heads, d)
    o, lse, got = gradients(s)
    ref, err = stored(s, o, lse, 2 if dtype == "f16" else p_terms)
    close(got, ref, err)


@pytest.mark.parametrize("spread", [6.0, 20.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_where_scores_are_large(spread, dtype):
    """Scores of hundreds and thousands: probabilities taken again from lse, whose rounding grows with its size."""
    s = tensors(36, TYPES[dtype], [60, 90, 1], [350, 500, 33], 2, 2, 128, spread=spread)
    o, lse, got = gradients(s)
    ref, err = stored(s, o, lse, 1)
    close(got, ref, err)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads,kv_heads,d,lq,lk", [(4, 2, 64, [33, 60], [54, 200]), (8, 2, 128, [1, 1, 1], [700, 40, 5000]), (3, 3, 30, [1, 2], [9, 90]),
                                                    (2, 1, 256, [100, 9], [300, 40])])
def test_outputs_of_few_rows_keep_both_terms(heads, kv_heads, d, lq, lk, dtype):
    """Up to 128 packed rows a tree: probabilities in two terms, so that an output is off by little more than its own rounding."""
    s = tensors(37, TYPES[dtype], lq, lk, heads, kv_heads, d)
    o, _ = binding.tl_attend(s["q"], s["k"], s["v"], with_lse=True, **where(s))
    h = half_step(TYPES[dtype]) if dtype != "f32" else 0.0
    a = b = 0
    for nq, nk in zip(lq, lk):
        rows, cols = slice(a, a + nq), slice(b, b + nk)
        a, b = a + nq, b + nk
        for j in range(heads):
            Q, K, V = s["q"][rows, j].double(), s["k"][cols, j * kv_heads // heads].double(), s["v"][cols, j * kv_heads // heads].double()
            S = Q @ K.t() * s["scale"]
            P = torch.softmax(S, 1)
            O = P @ V
            ds = (d + 4) * U * s["scale"] * (Q.abs() @ K.abs().t()).amax(1, keepdim=True)
            rel = 2 * ds + (8 * S.abs().amax(1, keepdim=True) + nk + 24) * U
            e = (rel + h * h + (2 * nk + 8) * U) * (P @ V.abs()) + (2.0 ** -39 if dtype == "f16" else 2.0 ** -125) * V.abs().sum(0)
            e = e + half_step(TYPES[dtype]) * (O.abs() + e) + (2.0 ** -25 if dtype == "f16" else 1e-36)
            bad = ~((o[rows, j].double() - O).abs() <= e)
            assert not bad.any(), (int(bad.sum()), float(((o[rows, j].double() - O).abs() / e).max()))
