"""Cross attention and its gradients against a plain implementation in 64 bits.

Bounds are worked out per element from the inputs (u = 2^-24, half a step of fp32; h = half a step of the operands' type):
  score       a sum of D products and three further roundings:                       |ds| <= (D + 4) u * scale * sum |q||k|
  probability exp of a difference of two scores, one rounding of each to base 2, a sum of n terms:
              relative 2 max|ds| + (4 max|s| + n + 12) u, and, where it is an operand of 16 bits, h (f16: 2^-25 absolute below its normal range)
  output      sum of n products of these with v: relative to sum P|v| that, and n u; rounded once to the type.
The gradients' bounds follow the same way from their formulas (see bounds()).
"""
import math

import numpy as np
import pytest
import torch

from paper_1809_00832_amd import binding

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def tensors(seed, dtype, lq, lk, heads, kv_heads, d, mask=0.0, packed=False, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    nq, nk = int(sum(lq)), int(sum(lk))
    new = lambda *s: (torch.randn(s, generator=g, device="cuda") * spread).to(dtype)
    if packed:                                               # rows of a wider projection, an odd number of elements apart where d is odd
        q = new(nq, heads + 1, d)[:, 1:]
        kv = new(nk, 2, kv_heads, d)
        k, v = kv[:, 0], kv[:, 1]
    else:
        q, k, v = new(nq, heads, d), new(nk, kv_heads, d), new(nk, kv_heads, d)
    m = None
    if mask:
        m = (torch.rand(nk, generator=g, device="cuda") >= mask).to(torch.uint8)
    return dict(q=q, k=k, v=v, q_off=offsets(lq), kv_off=offsets(lk), kv_mask=m, lq=lq, lk=lk, d_o=new(nq, heads, d), scale=d ** -0.5)


def plain(s, grads=True):
    """o, lse, d_q, d_k, d_v in 64 bits and a bound of the error of each."""
    q, k, v, g = (s[n].double() for n in ("q", "k", "v", "d_o"))
    dtype, scale = s["q"].dtype, s["scale"]
    G, D = q.shape[1] // k.shape[1], q.shape[2]
    h = half_step(dtype) if dtype != torch.float32 else 0.0
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    out = {n: torch.zeros_like(x) for n, x in (("o", q), ("d_q", q), ("d_k", k), ("d_v", v))}
    out["lse"] = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    err = {n: torch.zeros_like(x) for n, x in out.items()}
    a = b = 0
    for nq, nk in zip(s["lq"], s["lk"]):
        rows, cols = slice(a, a + nq), torch.arange(b, b + nk, device="cuda")
        a, b = a + nq, b + nk
        if s["kv_mask"] is not None:
            cols = cols[s["kv_mask"][cols] != 0]
        if nq == 0 or len(cols) == 0:
            continue
        n = len(cols)
        for j in range(q.shape[1]):
            Q, K, V, dO = q[rows, j], k[cols, j // G], v[cols, j // G], g[rows, j]
            S = Q @ K.t() * scale
            lse = torch.logsumexp(S, 1, keepdim=True)
            P = torch.exp(S - lse)
            O = P @ V
            ds = (D + 4) * U * scale * (Q.abs() @ K.abs().t()).amax(1, keepdim=True)
            rel = 2 * ds + (4 * S.abs().amax(1, keepdim=True) + n + 12) * U
            eo = (rel + h + n * U) * (P @ V.abs()) + tiny * V.abs().sum(0)
            out["o"][rows, j], err["o"][rows, j] = O, eo + half_step(dtype) * (O.abs() + eo)
            out["lse"][rows, j] = lse[:, 0]
            err["lse"][rows, j] = (rel + (4 + lse.abs()) * U)[:, 0]
            if not grads:
                continue
            # P is taken again from lse: its error comes in, and that of lse in base 2
            rel = 2 * rel + (8 + 4 * lse.abs()) * U
            e_o = eo + half_step(dtype) * (O.abs() + eo)
            delta = (dO * O).sum(1, keepdim=True)
            e_delta = (dO.abs() * e_o).sum(1, keepdim=True) + (D + 4) * U * (dO.abs() * (O.abs() + e_o)).sum(1, keepdim=True)
            dP = dO @ V.t()
            e_dP = (D + 4) * U * (dO.abs() @ V.abs().t())
            dS = P * (dP - delta)
            e_dS = rel * P * (dP - delta).abs() + P * (1 + rel) * (e_dP + e_delta + 2 * U * (dP - delta).abs())
            e_dS = e_dS + h * (dS.abs() + e_dS) + tiny
            m = nq * G
            dq, dk, dv = scale * dS @ K, scale * dS.t() @ Q, P.t() @ dO
            e_q = scale * (e_dS @ K.abs() + (n + 4) * U * (dS.abs() @ K.abs()))
            e_k = scale * (e_dS.t() @ Q.abs() + (m + 4) * U * (dS.abs().t() @ Q.abs()))
            e_v = (rel * P + h * P + tiny).t() @ dO.abs() + (m + 4) * U * (P.t() @ dO.abs())
            out["d_q"][rows, j], err["d_q"][rows, j] = dq, e_q + half_step(dtype) * (dq.abs() + e_q)
            out["d_k"][cols, j // G] += dk
            out["d_v"][cols, j // G] += dv
            err["d_k"][cols, j // G] += e_k
            err["d_v"][cols, j // G] += e_v
    for n in ("d_k", "d_v"):
        err[n] = err[n] + half_step(dtype) * (out[n].abs() + err[n])
    for n in ("o", "d_q", "d_k", "d_v"):                     # below the type's normal range steps no longer shrink
        err[n] = err[n] + (2.0 ** -25 if dtype == torch.float16 else 1e-36)
    return out, err


def where(s):
    return dict(q_off=s["q_off"], kv_off=s["kv_off"], kv_mask=s["kv_mask"], scale=s["scale"])


def call(s, grads=True):
    o, lse = binding.tl_attend(s["q"], s["k"], s["v"], with_lse=True, **where(s))
    out = {"o": o, "lse": lse}
    if grads:
        out.update(binding.tl_attend_backward(s["q"], s["k"], s["v"], o, lse, s["d_o"], **where(s)))
    return out


def close(got, ref, err, names=None):
    for n in names or got:
        x = got[n].double()
        same = (x == ref[n]) | ((x - ref[n]).abs() <= err[n])
        bad = int((~same).sum())
        assert bad == 0, "%s: %d of %d, worst %.3g times the bound" % (n, bad, same.numel(), float(((x - ref[n]).abs() / err[n].clamp(min=1e-300))[~same].max()))


SHORT_Q, LONG_Q = [3, 1, 0, 7, 2], [130, 257, 1, 200, 64]
SHORT_K, LONG_K = [1, 9, 33, 0, 64], [127, 128, 129, 300, 65]
SHAPES = [
    # heads, kv heads, d, queries, nodes, masked share, packed
    (1, 1, 1, SHORT_Q, SHORT_K, 0.0, False),
    (5, 5, 30, SHORT_Q, SHORT_K, 0.0, False),
    (5, 5, 30, LONG_Q, LONG_K, 0.3, True),
    (3, 1, 7, LONG_Q, SHORT_K, 0.3, True),
    (4, 4, 32, SHORT_Q, LONG_K, 0.3, False),
    (4, 2, 32, LONG_Q, LONG_K, 0.0, False),
    (8, 2, 64, [1] * 5, LONG_K, 0.0, True),
    (8, 8, 64, SHORT_Q, SHORT_K, 0.3, False),
    (4, 4, 64, LONG_Q, LONG_K, 0.0, True),
    (7, 1, 75, SHORT_Q, LONG_K, 0.3, False),
    (2, 2, 75, LONG_Q, LONG_K, 0.0, True),
    (4, 1, 128, [1] * 5, LONG_K, 0.3, False),
    (4, 1, 128, SHORT_Q, LONG_K, 0.0, True),
    (2, 1, 128, LONG_Q, LONG_K, 0.3, False),
    (2, 2, 129, SHORT_Q, LONG_K, 0.0, False),
    (2, 1, 200, LONG_Q, LONG_K, 0.3, False),
    (4, 2, 256, SHORT_Q, LONG_K, 0.3, False),
    (1, 1, 256, LONG_Q, LONG_K, 0.0, True),
]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_against_64_bits(case, dtype):
    heads, kv_heads, d, lq, lk, mask, packed = SHAPES[case]
    s = tensors(case, TYPES[dtype], lq, lk, heads, kv_heads, d, mask, packed)
    ref, err = plain(s)
    close(call(s), ref, err)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("lq,lk", [([1], [5001]), ([1, 2], [4096, 1]), ([3], [2049]), ([1, 0, 1], [3000, 3000, 0])])
def test_long_axis_of_few_queries(lq, lk, dtype):
    for heads, kv_heads, d in ((4, 1, 64), (2, 2, 128), (1, 1, 33), (2, 1, 256)):
        s = tensors(11, TYPES[dtype], lq, lk, heads, kv_heads, d, 0.25)
        ref, err = plain(s, grads=False)
        close(call(s, grads=False), ref, err, ["o", "lse"])


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_many_trees(dtype):
    rng = np.random.default_rng(3)
    lq, lk = rng.integers(0, 4, 4500).tolist(), rng.integers(0, 6, 4500).tolist()
    s = tensors(12, TYPES[dtype], lq, lk, 2, 1, 32, 0.2)
    ref, err = plain(s)
    close(call(s), ref, err)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("lq", [[1, 1, 1], [40, 40, 40], [300, 5, 100]])
@pytest.mark.parametrize("d", [30, 64, 128])
def test_what_masked_nodes_hold_has_no_effect(lq, d, dtype):
    """NaN, infinities and the type's extremes in rows that are not read; a tree whose every node is masked, beside others."""
    lk = [70, 45, 200]
    s = tensors(13, TYPES[dtype], lq, lk, 4, 2, d, 0.4, packed=True)
    s["kv_mask"][70:115] = 0
    clean = call(s)
    lim = torch.finfo(TYPES[dtype])
    for junk in (math.nan, math.inf, -math.inf, lim.min, lim.max):
        k, v = s["k"].clone(), s["v"].clone()
        k[s["kv_mask"] == 0] = junk
        v[s["kv_mask"] == 0] = junk
        got = call(dict(s, k=k, v=v))
        for n in clean:
            assert torch.equal(got[n], clean[n]), n
    rows = slice(lq[0], lq[0] + lq[1])
    assert not clean["o"][rows].any() and (clean["lse"][rows] == -math.inf).all() and not clean["d_q"][rows].any()
    off = s["kv_mask"] == 0
    assert not clean["d_k"][off].any() and not clean["d_v"][off].any()


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_no_value_crosses_into_another_tree(dtype):
    lq, lk = [5, 50, 3], [33, 70, 129]
    s = tensors(14, TYPES[dtype], lq, lk, 4, 2, 64)
    clean = call(s)
    bad = {n: s[n].clone() for n in ("q", "k", "v", "d_o")}
    bad["q"][5:55], bad["d_o"][5:55] = math.nan, math.inf
    bad["k"][33:103], bad["v"][33:103] = math.inf, math.nan
    got = call(dict(s, **bad))
    for n in clean:
        keep = [0, 1, 2, 3, 4, 55, 56, 57] if n in ("o", "lse", "d_q") else list(range(33)) + list(range(103, 232))
        assert torch.equal(got[n][keep], clean[n][keep]), n
    assert got["o"][5:55].isnan().all() and got["d_k"][33:103].isnan().all()


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_infinite_scores_follow_the_formula(dtype):
    """A row that meets +infinity is NaN, as softmax is; -infinity is a probability of zero; only -infinity gives zeros."""
    s = tensors(15, TYPES[dtype], [3], [40], 1, 1, 32)
    s["q"][:] = 0
    s["q"][0, 0, 0], s["q"][1, 0, 0] = 1, -1
    s["k"][:] = 0
    s["k"][7, 0, 0] = math.inf
    s["v"][:] = 1
    s["q"][2, 0, 1] = 1                                       # 0 * inf: NaN
    got = call(s, grads=False)
    assert got["o"][0].isnan().all() and (got["o"][1] == 1).all() and got["o"][2].isnan().all()
    s["k"][:, 0, 0] = math.inf
    s["q"][:, 0, 0] = -1
    s["q"][:, 0, 1] = 0
    s["k"][:, 0, 1:] = 0
    got = call(s)
    assert not got["o"].any() and (got["lse"] == -math.inf).all()


@pytest.mark.parametrize("spread", [8.0, 30.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(spread, dtype):
    """Scores of hundreds and thousands: the running maximum moves by more than exp can hold."""
    s = tensors(16, TYPES[dtype], [70, 3], [400, 300], 2, 1, 64, spread=spread)
    ref, err = plain(s, grads=False)
    got = call(s, grads=False)
    close(got, ref, err, ["o", "lse"])


def test_gradients_against_differences():
    s = tensors(17, torch.float32, [9, 40], [33, 65], 4, 2, 48, 0.2)
    got = call(s)
    g = torch.Generator(device="cuda").manual_seed(5)
    eps = 2.0 ** -12
    for name in ("q", "k", "v"):
        step = torch.randn(s[name].shape, generator=g, device="cuda", dtype=torch.float64)
        loss = []
        for sign in (1, -1):
            moved = dict(s, **{n: s[n].double() for n in ("q", "k", "v", "d_o")})
            moved[name] = moved[name] + sign * eps * step
            loss.append(float((plain(moved, grads=False)[0]["o"] * s["d_o"].double()).sum()))
        slope = (loss[0] - loss[1]) / (2 * eps)
        mine = float((got["d_" + name].double() * step).sum())
        # the third derivative's part of a central difference is of the order of eps^2 = 6e-8 of terms of order one; of the fp32 gradients'
        # errors, 2e-6 of their size each
        size = float((got["d_" + name].double().abs() * step.abs()).sum())
        assert abs(mine - slope) <= 1e-5 * size, (name, mine, slope, size)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_strides(dtype):
    """Heads in front of rows, rows and heads that repeat, outputs in place."""
    lq, lk = [20, 90], [50, 77]
    s = tensors(18, TYPES[dtype], lq, lk, 4, 2, 64, 0.2)
    ref = call(s)
    t = dict(s)
    for n in ("q", "k", "v", "d_o"):
        t[n] = s[n].transpose(0, 1).contiguous().transpose(0, 1)
    got = call(t)
    for n in ref:
        assert torch.equal(got[n], ref[n]), n
    o = torch.empty(4, 110, 64, dtype=TYPES[dtype], device="cuda").transpose(0, 1)
    assert binding.tl_attend(s["q"], s["k"], s["v"], o=o, **where(s)) is o and torch.equal(o, ref["o"])
    one = dict(s, k=s["k"][:, :1].expand(-1, 4, -1), v=s["v"][:, :1].expand(-1, 4, -1))       # one head of nodes, by stride 0 or by group
    shared = dict(s, k=s["k"][:, :1], v=s["v"][:, :1])
    a, b = call(one, grads=False), call(shared, grads=False)
    r, e = plain(shared, grads=False)
    close(a, r, e, ["o", "lse"])
    close(b, r, e, ["o", "lse"])
    # the same numbers at an address that only the element's size divides
    room = torch.empty(s["k"].numel() + 1, dtype=TYPES[dtype], device="cuda")
    room[1:] = s["k"].reshape(-1)
    got = call(dict(s, k=room[1:].view_as(s["k"])))
    for n in ref:
        assert torch.equal(got[n], ref[n]), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_beyond_32_bits(dtype):
    """Node rows so far apart that their offsets pass 2^32 elements."""
    size = torch.finfo(TYPES[dtype]).bits // 8
    step = (1 << 26) + 8
    nk = 70
    if torch.cuda.mem_get_info()[0] < 2 * step * nk * size:
        pytest.skip("not enough free device memory")
    store = torch.empty(step * nk, dtype=TYPES[dtype], device="cuda")
    s = tensors(19, TYPES[dtype], [3], [nk], 2, 1, 64)
    far = torch.as_strided(store, (nk, 1, 64), (step, 64, 1))
    far.copy_(s["k"])
    ref = call(s)
    got = call(dict(s, k=far))
    for n in ref:
        assert torch.equal(got[n], ref[n]), n


def test_nothing_to_do():
    z = lambda *s: torch.zeros(s, device="cuda")
    off0, off1 = offsets([]), offsets([0])
    for off in (off0, off1):
        assert binding.tl_attend(z(0, 2, 8), z(0, 1, 8), z(0, 1, 8), off, off).shape == (0, 2, 8)
    q, k = z(3, 2, 8) + 1, z(0, 1, 8)
    o, lse = binding.tl_attend(q, k, k, offsets([3]), off1, with_lse=True)
    assert not o.any() and (lse == -math.inf).all()
    g = binding.tl_attend_backward(q, k, k, o, lse, q, offsets([3]), off1)
    assert not g["d_q"].any() and g["d_k"].shape == (0, 1, 8)
    q, k = z(0, 2, 8), z(5, 1, 8) + 1
    o, lse = binding.tl_attend(q, k, k, off1, offsets([5]), with_lse=True)
    g = binding.tl_attend_backward(q, k, k, o, lse, q, off1, offsets([5]))
    assert not g["d_k"].any() and not g["d_v"].any()


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_repeats_bit_for_bit_on_any_stream(dtype):
    s = tensors(20, TYPES[dtype], [1, 130, 12], [3000, 257, 40], 8, 2, 64, 0.2)
    first = call(s)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        o, lse = binding.tl_attend(s["q"], s["k"], s["v"], with_lse=True, stream=other, **where(s))
        g = binding.tl_attend_backward(s["q"], s["k"], s["v"], o, lse, s["d_o"], stream=other, **where(s))
        other.synchronize()
        for n, x in dict(g, o=o, lse=lse).items():
            assert torch.equal(x, first[n]), n


@pytest.mark.parametrize("lq,lk", [([1] * 4, [3000] * 4), ([50, 90], [200, 77])])
def test_graph_replays(lq, lk):
    s = tensors(21, torch.bfloat16, lq, lk, 8, 2, 64, 0.2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(s)
    for seed in range(4):
        fresh = tensors(30 + seed, torch.bfloat16, lq, lk, 8, 2, 64)
        for n in ("q", "k", "v", "d_o"):
            s[n].copy_(fresh[n])
        want = {n: x.clone() for n, x in call(s).items()}
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(out[n], want[n]), n


def test_an_encoders_states_are_read_and_given_gradients():
    """Attention over the states of an evaluated batch; the gradient arrives at the encoder's parameters.  Against differences of the loss
    in the encoder's own states (64 bits), and tl_backward takes the rows as they are."""
    from paper_1809_00832_amd import synth
    w = synth.workload("tiny")
    net = binding.TreeNet(w.params, scheduler="level_device")
    batch = net.load(w.trees)
    binding.tl_set_keep_gates(net.ctx, True)
    net.forward()
    H = w.params.hidden
    lk = np.diff(w.trees.tree_off).tolist()
    lq = [2] * len(lk)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(sum(lq), 1, H, generator=g, device="cuda")
    states = batch["h"].view(-1, 1, H)
    s = dict(q=q, k=states, v=states, q_off=offsets(lq), kv_off=batch["tree_off"], kv_mask=None, lq=lq, lk=lk, scale=0.25,
             d_o=torch.randn(q.shape, generator=g, device="cuda"))
    ref, err = plain(s)
    got = call(s)
    close(got, ref, err)
    g_h = (got["d_k"] + got["d_v"]).view(-1, H).contiguous()
    grads = binding.tl_backward(net.ctx, batch, g_h, w.params.embed_dim)
    assert grads["d_u"].isfinite().all() and grads["d_u"].any()
    net.close()


@pytest.mark.parametrize("size", [2.0 ** -14, 1.0, 2.0 ** 10])
def test_fp16_gradients_of_any_size(size):
    """Score gradients as operands of 16 bits: upstream gradients near the type's least normal value, and large ones of a scaled loss, beside rows a
    thousand times smaller in another tree.  The bound is that of test_against_64_bits; gradients whose values fp16 cannot hold are left out."""
    s = tensors(22, torch.float16, [40, 3, 150], [50, 70, 90], 4, 2, 64, 0.2)
    s["d_o"] = (s["d_o"].float() * size).half()
    s["d_o"][40:43] *= 2.0 ** -6
    ref, err = plain(s)
    got = call(s)
    for n in got:
        fits = ref[n].abs() < 6e4
        assert fits.float().mean() > 0.99
        x = got[n].double()
        bad = fits & (x != ref[n]) & ~((x - ref[n]).abs() <= err[n])
        assert not bad.any(), n


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("lq,lk", [([2], [5001]), ([1100], [3]), ([3, 0, 900, 1], [4000, 50, 2, 0]), ([600, 2], [700, 2500])])
def test_gradients_of_few_trees(lq, lk, dtype):
    """Sums over many nodes, or over many rows, of few trees: divided among workgroups, joined by a second launch; masked nodes among them."""
    for heads, kv_heads, d, mask in ((2, 2, 64, 0.0), (4, 1, 128, 0.25), (3, 1, 33, 0.25), (1, 1, 256, 0.0)):
        s = tensors(23, TYPES[dtype], lq, lk, heads, kv_heads, d, mask)
        ref, err = plain(s)
        got = call(s)
        close(got, ref, err)
        for n, x in call(s).items():
            assert torch.equal(x, got[n]), n


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads,kv_heads,d,mask", [(2, 2, 64, 0.0), (6, 2, 33, 0.0), (3, 1, 128, 0.3), (1, 1, 256, 0.3)])
def test_a_long_tree_among_short_ones(heads, kv_heads, d, mask, dtype):
    """Short trees on average, so that LDS holds one stage at a time, and trees among them that need many stages of nodes and of rows."""
    lq, lk = [3, 1, 0, 2] * 12, [9, 1, 13, 0] * 12
    lq[5], lk[5] = 2, 500
    lq[21], lk[21] = 260, 7
    lq[40], lk[40] = 150, 333
    s = tensors(24, TYPES[dtype], lq, lk, heads, kv_heads, d, mask)
    ref, err = plain(s)
    got = call(s)
    close(got, ref, err)
    for n, x in call(s).items():
        assert torch.equal(x, got[n]), n
