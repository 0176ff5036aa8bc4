"""The recurrence where products of gates leave the range of fp32, or states do on the way: outputs are those of the loop over the words.

The reference is that loop: every word's value is taken in 64 bits (products of fp32 numbers are exact there) and rounded to fp32, subnormal numbers kept, overflow to
infinity.  Bounds, u = 2^-24: a word is met to 4 u of its magnitude M_t = |f_t| M_(t-1) + |i_t x_t| (sigmoid gates: (2 |g| + 12) u), and to 2^-120 of the largest magnitude S_t so far: the
product of n gates is rounded to multiples of 2^-149 where it is subnormal, so that a state s is met to n 2^-149 |s| behind them, with n up to 2^10 gates of parts joined at once and products up to
2^16 of what was joined before: 2^-123, and again where a wave's own run follows.  So E_t = |f_t| E_(t-1) + d_t M_t + 2^-120 S_t, and a step of 2^-149 for what is subnormal itself.  What goes back likewise.  fp32 throughout, so nothing is rounded to fewer bits.
A sigmoid gate below 2^-126 is zero.
"""
import numpy as np
import pytest
import torch

from paper_1809_00832_amd import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SIGMOID, GIVEN = binding.TL_GATE_SIGMOID, binding.TL_GATE_GIVEN
STEP, LEAST = 2.0 ** -120, 2.0 ** -149


def f32(v):
    return v.astype(np.float32).astype(np.float64)


@np.errstate(all="ignore")
def loop(g, x, h0, gate, d_h, d_last):
    """One sentence: outputs, bounds of their errors, and the magnitudes that decide whether a word is too near to the largest number to be told."""
    if gate == GIVEN:
        f, i, d = g, np.ones_like(g), np.full_like(g, 4 * U)
    else:
        f, i, d = f32(1 / (1 + np.exp(-g))), f32(1 / (1 + np.exp(g))), (2 * np.abs(g) + 12) * U
        f, i = np.where(f < 2.0 ** -126, 0.0, f), np.where(i < 2.0 ** -126, 0.0, i)
    L, C = g.shape
    out = {k: np.zeros((L, C)) for k in ("h", "d_g", "d_x")}
    err, near = {k: np.zeros((L, C)) for k in out}, np.zeros((L, C), dtype=bool)
    h, m, e = h0.copy(), np.abs(h0), np.zeros(C)
    top = m.copy()
    before, before_m, before_e = np.zeros((L, C)), np.zeros((L, C)), np.zeros((L, C))
    edge = lambda v: (np.abs(v) > 2.0 ** 127.99) & (np.abs(v) < 2.0 ** 128.01)
    for t in range(L):
        before[t], before_m[t], before_e[t] = h, m, e
        wide = f[t] * h + f32(i[t] * x[t])
        near[t] |= edge(wide)
        h = f32(wide)
        m = np.abs(f[t]) * m + np.abs(i[t] * x[t])
        top = np.maximum(top, m)
        e = np.abs(f[t]) * e + d[t] * m + STEP * top + LEAST
        out["h"][t], err["h"][t] = h, e
    back, m, e = d_last.copy(), np.abs(d_last), np.zeros(C)
    top = m.copy()
    for t in range(L - 1, -1, -1):
        wide = back + d_h[t]
        near[t] |= edge(wide)
        lam, lam_m = f32(wide), m + np.abs(d_h[t])
        lam_e = e + 2 * U * lam_m
        out["d_x"][t], err["d_x"][t] = f32(lam * i[t]), i[t] * lam_e + (d[t] + 2 * U) * np.abs(i[t]) * lam_m + LEAST
        near[t] |= edge(lam * i[t])
        back = f32(lam * f[t])
        near[t] |= edge(lam * f[t])
        if gate == SIGMOID:
            rest, by, own = f32(before[t] - x[t]), f[t] * i[t], f32(back * i[t])
            rest_m = before_m[t] + np.abs(x[t])
        else:
            rest, by, own, rest_m = before[t], np.ones(C), lam, before_m[t]
        out["d_g"][t] = f32(own * rest)
        near[t] |= edge(own * rest)
        err["d_g"][t] = by * (lam_e * np.abs(rest) + lam_m * before_e[t] + (2 * d[t] + 8 * U) * lam_m * rest_m) + LEAST * (2 + np.abs(rest) + rest_m)
        top = np.maximum(top, lam_m)
        m, e = np.abs(f[t]) * lam_m, np.abs(f[t]) * lam_e + d[t] * np.abs(f[t]) * lam_m + STEP * top + LEAST
    out["h_last"], err["h_last"], out["d_h0"], err["d_h0"] = h[None], err["h"][-1:], back[None], e[None]
    near_back = np.flip(np.maximum.accumulate(np.flip(near, 0), 0), 0) | np.maximum.accumulate(near, 0)
    return out, err, near_back


def check(g, x, h0, gate, d_h, d_last):
    """All sentences of one length, side by side as channels are: g, x [L, C] (CUDA, fp32)."""
    L = g.shape[0]
    off = torch.tensor([0, L], dtype=torch.int32, device="cuda")
    got = binding.tl_recur(g, x, off, h0, gate, with_last=True, with_tape=True)
    tape = got.pop("tape")
    got.update(binding.tl_recur_backward(g, x, off, tape, d_h, d_last, gate))
    H = lambda t: t.double().cpu().numpy()
    want, err, near = loop(H(g), H(x), H(h0)[0], gate, H(d_h), H(d_last)[0])
    for k, v in got.items():
        a, w, e = H(v), want[k], err[k]
        skip = near if k in ("h", "d_g", "d_x") else near.any(0)[None]
        with np.errstate(invalid="ignore"):
            same = (a == w) | (np.isnan(a) & np.isnan(w)) | (np.isfinite(a) & np.isfinite(w) & (np.abs(a - w) <= 1.01 * e)) | skip
        assert same.all(), (k, np.argwhere(~same)[:4].tolist(), a[~same][:4], w[~same][:4], e[~same][:4])


def zeros(L, C):
    z = lambda *s: torch.zeros(s, device="cuda")
    return z(L, C), z(L, C), z(1, C), z(L, C), z(1, C)


LENGTHS = [1, 4, 8, 30, 64, 130, 300, 1500, 9000]


@pytest.mark.parametrize("L", LENGTHS)
def test_products_that_vanish_and_come_back(L):
    """Small gates first, then large ones: the product of all is one, that of the first ones is zero in fp32."""
    C = 12
    g, x, h0, d_h, d_last = zeros(L, C)
    g += 1
    h0 += 1e35
    d_last += 1e35
    pattern = [1e-30, 1e-30, 1e30, 1e30]
    for c in range(8):                          # wherever runs begin
        for k, v in enumerate(pattern):
            if c + k < L:
                g[c + k, c] = v
            if L - 1 - c - k >= 0 and c % 2:
                g[L - 1 - c - k, c] = v         # ... and from behind, as gradients pass them
    n = L // 5                                  # a fifth of the sentence whose product is 1e-60, another one that brings it back
    if n > 1:
        g[n:2 * n, 8], g[3 * n:4 * n, 8] = 10.0 ** (-60 / n), 10.0 ** (60 / n)
        g[n:2 * n, 9], g[3 * n:4 * n, 9] = 10.0 ** (-44 / n), 10.0 ** (44 / n)
    h0[0, 9], d_last[0, 9] = 3.0, 5.0
    g[:, 10] = 10.0 ** (-50 / max(L, 2))
    g[::2, 11], g[1::2, 11] = -1e-25, -1e25
    check(g, x, h0, GIVEN, d_h, d_last)


@pytest.mark.parametrize("L", LENGTHS)
def test_states_that_overflow_between(L):
    """Infinite in the loop from some word on, finite by the product of the gates."""
    C = 10
    g, x, h0, d_h, d_last = zeros(L, C)
    g += 1
    h0 += 1e30
    d_last += 1e30
    for c in range(4):
        if L >= c + 2:
            g[c, c], g[c + 1, c] = 1e30, 1e-30
            g[L - 1 - c, 4 + c], g[L - 2 - c, 4 + c] = 1e30, 1e-30
    x[L // 2, 8], h0[0, 8] = 3e38, 3e38         # one sum of two words overflows
    g[L // 2 + 1:, 8] = 1e-3
    d_h[L // 2, 9], d_last[0, 9] = 3e38, 3e38
    g[:L // 2 + 1, 9] = 1e-3
    check(g, x, h0, GIVEN, d_h, d_last)


@pytest.mark.parametrize("L", LENGTHS)
def test_sigmoid_gates_whose_product_vanishes(L):
    """Large states and gradients that decay to numbers of ordinary size, by a product that fp32 does not hold; gradients that overflow on the way."""
    C = 7
    g, x, h0, d_h, d_last = zeros(L, C)
    h0 += 1e35
    d_last += 1e35
    for c, decades in enumerate((40, 46, 60)):
        p = 10.0 ** (-decades / L)
        g[:, c] = float(np.log(p / (1 - p)))
    g[:, 3] = -13.0
    g[:, 4] = -13.0
    d_h[L // 2, 4], d_last[0, 4] = 3e38, 0.0
    g[:, 5], g[L // 2:, 5] = -6.9, 20.0
    d_h[L // 2, 5], d_last[0, 5] = 3e38, 3e38   # lambda overflows at one word: all before it are infinite
    g[L // 2, 6], g[L // 2 + 1:, 6] = -200.0, 1.0          # a gate that is zero
    check(g, x, h0, SIGMOID, d_h, d_last)


@pytest.mark.parametrize("L", [8, 40, 200, 700, 3000])
@pytest.mark.parametrize("spread", [0.3, 3.0, 30.0])
def test_gates_of_any_magnitude(L, spread):
    """Gates of either sign whose magnitudes are spread over some or many powers of ten, some of them zero; inputs and first states likewise."""
    C = 96
    rng = np.random.default_rng(L * 1000 + int(spread * 10))
    new = lambda *s: torch.from_numpy((rng.choice([-1.0, 1.0], s) * 10.0 ** rng.normal(0, spread, s).clip(-37, 37)).astype(np.float32)).cuda()
    g, x, h0, d_h, d_last = new(L, C), new(L, C), new(1, C), new(L, C), new(1, C)
    walk = np.cumsum(np.log10(np.abs(g.double().cpu().numpy())), 0)
    g[:, :48] *= torch.from_numpy(10.0 ** -np.diff(np.concatenate([np.zeros((1, 48)), np.floor(walk[:, :48] / 30) * 30]), axis=0).clip(-37, 37)).float().cuda()   # products that come back
    x[:, 24:72] = 0.0
    d_h[:, 24:72] = 0.0
    g[torch.from_numpy(rng.random((L, C)) < 0.02).cuda()] = 0.0
    check(g, x, h0, GIVEN, d_h, d_last)


@pytest.mark.parametrize("L", [64, 700, 3000])
def test_open_and_closed_gates_of_ordinary_words(L):
    """Channels without inputs, words that are closed at once, and states above one that fade: ordinary numbers, products that vanish."""
    C = 70
    gen = torch.Generator(device="cuda").manual_seed(L)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda")
    g, x, h0, d_h, d_last = new(L, C) * 8, new(L, C), new(1, C) * 4, new(L, C), new(1, C) * 4
    x[:, ::3], d_h[:, ::4] = 0.0, 0.0
    check(g, x, h0, SIGMOID, d_h, d_last)
    g = torch.rand(L, C, generator=gen, device="cuda") ** 8
    g[torch.rand(L, C, generator=gen, device="cuda") < 0.05] = 0.0
    check(g, x, h0, GIVEN, d_h, d_last)


@pytest.mark.parametrize("lengths", [[40] * 30, [700, 900]], ids=["whole", "parts"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_channels_do_not_depend_on_one_another(dtype, lengths):
    """Gates above one, infinite ones, large states and gradients in some channels: the others keep their bits."""
    n, C = sum(lengths), 131
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s, dt=dtype: torch.randn(s, generator=gen, device="cuda", dtype=dt)
    g, x, d_h = new(n, C).tanh(), new(n, C), new(n, C)
    h0, d_last = new(len(lengths), C, dt=torch.float32), new(len(lengths), C, dt=torch.float32)
    off = torch.tensor([0] + lengths, device="cuda").cumsum(0).int()

    def run():
        out = binding.tl_recur(g, x, off, h0, GIVEN, with_last=True, with_tape=True)
        return dict(out, **binding.tl_recur_backward(g, x, off, out.pop("tape"), d_h, d_last, GIVEN))

    before = run()
    g[::3, 4], g[7, 20], g[9, 130], h0[:, 37], d_h[:, 60], x[5, 90] = 1.5, float("inf"), -1e30, 1e20, 1e15, float("nan")
    after = run()
    own = torch.ones(C, dtype=torch.bool, device="cuda")
    own[[4, 20, 130, 37, 60, 90]] = False
    for k in before:
        assert torch.equal(before[k][:, own], after[k][:, own]), k
        assert not torch.equal(before[k][:, 4], after[k][:, 4]), k


@pytest.mark.parametrize("L", [100, 900, 5000])
def test_large_states_and_gradients_of_gates_up_to_one(L):
    """Sums along the sentence, of numbers far above 2^40, and states that fade from there to ordinary numbers and on."""
    C = 40
    gen = torch.Generator(device="cuda").manual_seed(L)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda")
    g, x, h0, d_h, d_last = torch.ones(L, C, device="cuda"), new(L, C) * 1e20, new(1, C) * 1e25, new(L, C) * 1e18, new(1, C) * 1e22
    g[:, 10:20] = 1 - torch.rand(L, 10, generator=gen, device="cuda") ** 3
    g[:, 20:30] *= -1
    x[:, 25:], d_h[:, 25:] = 0.0, 0.0
    g[:, 30:35] = 10.0 ** (-70 / L)
    g[:, 35:] = torch.rand(L, 5, generator=gen, device="cuda") ** 4
    check(g, x, h0, GIVEN, d_h, d_last)
