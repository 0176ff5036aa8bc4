"""Waits between the parts of divided sentences that run out: the words are walked instead, and results are the loop's.

spin_limit bounds a wait's polls: with -1 nobody waits and every part but a sentence's first one walks, with 1 and 3 some do, by chance of the moment.  Inputs, reference and bounds
are those of test_gpu_recur: a walk is the loop that they are made of.
"""
import numpy as np
import pytest
import torch

from paper_1809_00832_amd import binding
from test_gpu_recur import GIVEN, SIGMOID, TYPES, check, host, inputs, offsets, reference

pytestmark = pytest.mark.gpu


def divided(g, off, back):
    r = binding._recurrence(g, g, off, SIGMOID, 0)
    return binding._recur_workspace(r, back, g.device)[1] > 0


# (a sentence of more than 32 parts of 128 or 64 words: a state that is handed on; empty sentences; parts that end early)
LENGTHS = {"two": [300, 200], "ragged": [700, 0, 1, 650, 64, 0], "states": [4500, 0]}


@pytest.mark.parametrize("spin_limit", [-1, 1, 3])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("gate", [SIGMOID, GIVEN], ids=["sigmoid", "given"])
@pytest.mark.parametrize("dtype,C", [("f32", 70), ("bf16", 37), ("f16", 130)])
def test_states_and_gradients(dtype, C, gate, lengths, spin_limit):
    lengths = LENGTHS[lengths]
    g, x, h0, d_h, d_last = inputs(lengths, C, TYPES[dtype], gate, seed=C)
    off = offsets(lengths)
    assert divided(g, off, 0) and divided(g, off, 1)
    state = h0.clone()
    out = binding.tl_recur(g, x, off, state, gate, h_last=state, with_tape=True, spin_limit=spin_limit)          # (in place of the first states)
    out.update(binding.tl_recur_backward(g, x, off, out["tape"], d_h, d_last, gate, spin_limit=spin_limit))
    want, err = reference(host(g), host(x), lengths, host(h0), gate, host(d_h), host(d_last))
    check(out, want, err, TYPES[dtype], sum(lengths))


@pytest.mark.parametrize("spin_limit", [-1, 1])
def test_large_parts_without_first_states(spin_limit):
    """Sentences that are cut into large parts, h0 and d_last zero: against the same call with its waits, each side within the bounds of the loop."""
    lengths, C = [3000, 3500], 2050
    g, x, _, d_h, _ = inputs(lengths, C, torch.bfloat16, SIGMOID, seed=4)
    off = offsets(lengths)

    def both(**kw):
        out = binding.tl_recur(g, x, off, None, with_last=True, with_tape=True, **kw)
        return dict(out, **binding.tl_recur_backward(g, x, off, out["tape"], d_h, None, **kw))

    got, want = both(spin_limit=spin_limit), both()
    some = np.random.default_rng(0).choice(C, 24, replace=False)
    ref, err = reference(host(g)[:, some], host(x)[:, some], lengths, None, SIGMOID, host(d_h)[:, some], np.zeros((2, 24)))
    for out in (got, want):
        check({k: out[k][:, torch.from_numpy(some).cuda()] for k in ("h", "h_last", "d_g", "d_x", "d_h0")}, ref, err, torch.bfloat16, sum(lengths))
    for k in ("h", "d_g", "d_x"):                       # (every channel: a step or two of the type where the last bits of a state differ, and 2^-10 of the magnitudes around)
        a, b = got[k].float(), want[k].float()
        assert ((a - b).abs() <= 2.0 ** -6 * b.abs() + 2.0 ** -10).all(), k


def test_infinities_and_nan():
    """Walked words have infinities and NaN where the loop has them, and other channels keep to themselves."""
    L, C = 700, 12
    g, x, h0, d_h, d_last = inputs([L], C, torch.float32, SIGMOID, seed=2)
    x[200, 1], x[300, 2], h0[0, 3], d_h[500, 4], d_last[0, 5] = float("inf"), float("nan"), -float("inf"), float("nan"), float("inf")
    off = offsets([L])
    out = binding.tl_recur(g, x, off, h0, with_last=True, with_tape=True, spin_limit=-1)
    h = out["h"]
    assert torch.isfinite(h[:200, 1]).all() and (h[200:, 1] == float("inf")).all() and torch.isfinite(h[:300, 2]).all() and torch.isnan(h[300:, 2]).all()
    assert (h[:, 3] == -float("inf")).all() and torch.isfinite(h[:, [0, 4, 5, 6, 7, 8, 9, 10, 11]]).all()
    d = binding.tl_recur_backward(g, x, off, out["tape"], d_h, d_last, spin_limit=-1)["d_x"]
    assert torch.isfinite(d[501:, 4]).all() and torch.isnan(d[:501, 4]).all() and (d[:, 5] == float("inf")).all()
    assert torch.isfinite(d[:, [0, 6, 7, 8, 9, 10, 11]]).all()


def test_any_limit_is_taken():
    lengths = [500, 400]
    g, x, h0, _, _ = inputs(lengths, 20, torch.float32, SIGMOID)
    off = offsets(lengths)
    want = binding.tl_recur(g, x, off, h0, with_last=True)
    for spin_limit in (2 ** 31 - 1, 1 << 16, 1 << 20):
        got = binding.tl_recur(g, x, off, h0, with_last=True, spin_limit=spin_limit)
        assert all(torch.equal(got[k], want[k]) for k in want)
    walked = binding.tl_recur(g, x, off, h0, spin_limit=-2 ** 31)["h"]
    assert ((walked - want["h"]).abs() <= 1e-4).all()
