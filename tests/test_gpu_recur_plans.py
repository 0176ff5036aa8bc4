"""Each way in which sentences are divided, for all types and gates, against the loop over the words in 64 bits (on the device, all sentences side by side).

Bounds are those of test_gpu_recur: u = 2^-24, a sigmoid gate to (2 |g| + 12) u, a given one's product and sum to 4 u; M_t = |f_t| M_(t-1) + |i_t x_t|, E_t = |f_t| E_(t-1) + d_t M_t; half a
step of the type where something is stored; and 2^-80, far above the 2^-120 of a state that a vanished product loses.
"""
import numpy as np
import pytest
import torch

from paper_1809_00832_amd import binding
from test_gpu_recur import GIVEN, SIGMOID, TYPES, U, inputs, offsets

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -80
BOTH = pytest.mark.parametrize("gate", [SIGMOID, GIVEN], ids=["sigmoid", "given"])


def reference(g, x, lengths, h0, gate, d_h, d_last):
    """Outputs in 64 bits and bounds of their errors before they are stored."""
    n, C = g.shape
    L = torch.tensor(lengths, device="cuda")
    order = torch.argsort(L, descending=True)
    live = (L[order][None, :] > torch.arange(max(lengths), device="cuda")[:, None]).sum(1).tolist()
    at = (torch.cumsum(L, 0) - L)[order]
    new = lambda: torch.zeros(n, C, dtype=torch.float64, device="cuda")
    out, err, before, before_m, before_e = {}, {}, new(), new(), new()
    for k in ("h", "d_g", "d_x"):
        out[k], err[k] = new(), new()
    h = torch.zeros(len(lengths), C, dtype=torch.float64, device="cuda") if h0 is None else h0.double()[order]
    m, e = h.abs(), torch.zeros_like(h)

    def gates(rows):
        v = g[rows].double()
        if gate == GIVEN:
            return v, torch.ones_like(v), torch.full_like(v, 4 * U)
        return torch.sigmoid(v), torch.sigmoid(-v), (2 * v.abs() + 12) * U

    for t, k in enumerate(live):
        rows = at[:k] + t
        f, i, d = gates(rows)
        u = i * x[rows].double()
        before[rows], before_m[rows], before_e[rows] = h[:k], m[:k], e[:k]
        h[:k] = f * h[:k] + u
        m[:k] = f.abs() * m[:k] + u.abs()
        e[:k] = f.abs() * e[:k] + d * m[:k] + STEP
        out["h"][rows], err["h"][rows] = h[:k], e[:k]
    back = torch.argsort(order)
    out["h_last"], err["h_last"] = h[back], e[back]
    lam = d_last.double()[order]
    m, e = lam.abs(), torch.zeros_like(lam)
    for t in range(len(live) - 1, -1, -1):
        k = live[t]
        rows = at[:k] + t
        f, i, d = gates(rows)
        here, here_m = lam[:k] + d_h[rows].double(), m[:k] + d_h[rows].double().abs()
        here_e = e[:k] + 2 * U * here_m
        out["d_x"][rows], err["d_x"][rows] = here * i, i * (here_e + (d + 2 * U) * here_m) + STEP
        rest, rest_m, by = before[rows], before_m[rows], torch.ones_like(f)
        if gate == SIGMOID:
            w = x[rows].double()
            rest, rest_m, by = rest - w, rest_m + w.abs(), f * i
        out["d_g"][rows] = here * rest * by
        err["d_g"][rows] = by * (here_e * rest.abs() + here_m * before_e[rows] + (2 * d + 8 * U) * here_m * rest_m) + STEP * (1 + rest_m + here_m)
        lam[:k], m[:k], e[:k] = f * here, f.abs() * here_m, f.abs() * here_e + d * f.abs() * here_m + STEP
    out["d_h0"], err["d_h0"] = lam[back], e[back]
    return out, err


def half_step(dtype, value):
    tiny = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}[dtype]
    return value.abs() * (torch.finfo(dtype).eps / 2) + tiny


def check(lengths, C, dtype, gate, first=True, packed=False, seed=0):
    dtype = TYPES[dtype]
    g, x, h0, d_h, d_last = inputs(lengths, C, dtype, gate, seed=seed, packed=packed, first=first)
    off = offsets(lengths)
    out = binding.tl_recur(g, x, off, h0, gate, with_last=True, with_tape=True)
    out.update(binding.tl_recur_backward(g, x, off, out.pop("tape"), d_h, d_last, gate))
    want, err = reference(g, x, lengths, h0, gate, d_h, d_last)
    for k, v in out.items():
        e = err[k]
        if k in ("h", "d_g", "d_x"):
            e = e + half_step(dtype, want[k]) + half_step(dtype, e)
        bad = (v.double() - want[k]).abs() - 1.01 * e
        assert v.shape == want[k].shape and bool((bad <= 0).all()), (k, float(bad.max()), torch.nonzero(bad > 0)[:4].tolist())
    # states alone (which are read past the caches), in place of the first ones
    state = torch.zeros_like(d_last) if h0 is None else h0.clone()
    alone = binding.tl_recur(g, x, off, state, gate, h_last=state)
    if h0 is not None:
        assert torch.equal(alone["h"], out["h"]) and torch.equal(state, out["h_last"])
    else:
        assert bool(((state.double() - want["h_last"]).abs() <= 1.01 * err["h_last"]).all())


def workspace(lengths, C, dtype, back):
    g = torch.empty(sum(lengths), C, dtype=TYPES[dtype], device="cuda")
    return binding._recur_workspace(binding._recurrence(g, g, offsets(lengths), SIGMOID, 0), back, g.device)[1]


def parts_of(lengths, C, dtype, back):
    """Words of a part, by the workspace's size (0: sentences are whole): pairs, states behind every 32nd part and a line of each slice, a table of parts, first states."""
    size = workspace(lengths, C, dtype, back)
    if size == 0:
        return 0
    up = lambda n: -(-n // 16) * 16
    lane = 1 if dtype == "f32" or C == 1 else 2
    for shift in (8, 7, 6):
        slots = (sum(lengths) >> shift) + len(lengths)
        if size == up(8 * slots * C) + up(4 * ((slots // 32 + 1) * C + 32 * -(-C // (64 * lane)))) + 16 * slots + (0 if back else up(4 * len(lengths) * C)) + 16:
            return 1 << shift
    raise AssertionError("parts of no known size")


def units():
    return torch.cuda.get_device_properties(0).multi_processor_count


RNG = np.random.default_rng(11)
# more than eight workgroups a unit, 8 to 32 words a sentence on average; some end within a block, some take several (32 words forwards, 64 backwards)
BRIEF = [int(v) for v in RNG.integers(0, 45, 2100)]
BRIEF[:12] = [64, 65, 63, 128, 129, 200, 31, 32, 33, 0, 1, 190]
PARTS = [int(v) for v in RNG.integers(1500, 1800, 8)]


@BOTH
@pytest.mark.parametrize("dtype,C", [("f32", 37), ("f32", 65), ("bf16", 37), ("bf16", 130), ("f16", 37), ("f16", 1)])
def test_many_brief_sentences(dtype, C, gate):
    mean = sum(BRIEF) / len(BRIEF)
    assert 8 < mean <= 32 and len(BRIEF) >= 8 * units() and workspace(BRIEF, C, dtype, 0) == workspace(BRIEF, C, dtype, 1) == 0
    check(BRIEF, C, dtype, gate, packed=C == 37)


@BOTH
@pytest.mark.parametrize("dtype,C", [("f32", 451), ("bf16", 901), ("f16", 902)])
def test_large_parts(dtype, C, gate):
    assert parts_of(PARTS, C, dtype, 0) == 256 and parts_of(PARTS, C, dtype, 1) == 128
    check(PARTS, C, dtype, gate, packed=dtype == "bf16")


@pytest.mark.parametrize("dtype,C,gate", [("bf16", 1501, SIGMOID), ("f16", 1500, GIVEN)])
def test_more_than_32_large_parts(dtype, C, gate):
    """States that are handed on behind every 32nd part, in both directions."""
    lengths = [8700, 9300]
    assert parts_of(lengths, C, dtype, 0) == 256 and parts_of(lengths, C, dtype, 1) == 128
    check(lengths, C, dtype, gate, first=False)


@BOTH
@pytest.mark.parametrize("dtype,C", [("f32", 100), ("bf16", 129), ("f16", 127), ("bf16", 1), ("f32", 1)])
def test_small_parts(dtype, C, gate):
    lengths = [900, 0, 1300, 1, 129]
    assert parts_of(lengths, C, dtype, 0) == 128 and parts_of(lengths, C, dtype, 1) == 64
    check(lengths, C, dtype, gate)


@BOTH
@pytest.mark.parametrize("dtype,C", [("f32", 130), ("bf16", 255), ("f16", 64)])
def test_whole_sentences(dtype, C, gate):
    lengths = [int(v) for v in np.random.default_rng(3).integers(0, 180, 90)]
    assert sum(lengths) > 32 * len(lengths) and workspace(lengths, C, dtype, 0) == 0
    check(lengths, C, dtype, gate, packed=True)


@BOTH
@pytest.mark.parametrize("dtype,C", [("f32", 130), ("bf16", 255), ("f16", 64)])
def test_a_few_words_each(dtype, C, gate):
    """One wave a sentence forwards, some of several blocks of eight words."""
    lengths = [int(v) for v in np.random.default_rng(4).integers(0, 14, 300)]
    lengths[:3] = [8, 9, 70]
    assert sum(lengths) <= 8 * len(lengths)
    check(lengths, C, dtype, gate)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_nan_stays_in_its_channel_and_sentence_of_large_parts(dtype):
    C = 901
    g, x, h0, d_h, d_last = inputs(PARTS, C, TYPES[dtype], SIGMOID)
    off = offsets(PARTS)
    assert parts_of(PARTS, C, dtype, 0) == 256

    def all_of(x, d_h):
        out = binding.tl_recur(g, x, off, h0, with_last=True, with_tape=True)
        return dict(out, **binding.tl_recur_backward(g, x, off, out.pop("tape"), d_h, d_last))

    a, b = sum(PARTS[:3]), sum(PARTS[:4])
    r = a + 700
    bad, bad_d = x.clone(), d_h.clone()
    bad[r, 899] = float("nan")
    bad_d[r, 900] = float("nan")
    clean, got = all_of(x, d_h), all_of(bad, bad_d)
    for k, want in clean.items():
        touched = torch.zeros_like(want, dtype=torch.bool)
        if k == "h":
            touched[r:b, 899] = True
        elif k == "h_last":
            touched[3, 899] = True
        elif k == "d_g":
            touched[r:b, 899] = True
            touched[a:r + 1, 900] = True
        elif k == "d_x":
            touched[a:r + 1, 900] = True
        else:
            touched[3, 900] = True
        assert torch.isnan(got[k][touched]).all() and torch.equal(got[k][~touched], want[~touched]), k
