"""Timed cases of what a sentence decoder needs between its attention and its update: a state that runs along the words, dropout, and
the words' log probabilities with their gradient.

A decoder that writes sentences from trees (perf/operators.py has its attention and its sampling) carries a state from word to word,
is trained with dropout on the cross entropy of given sentences, and scores given sentences.

Kinds of call:
  token    tl_recur with one row per sentence: the state's next step (serving)
  scan     tl_recur over whole sentences: scoring, a prompt
  train    tl_recur and tl_recur_backward: states and the gradients of gates, inputs and first states
  rank     tl_score: log probabilities of given words, entropies, and the most probable words beside them
  loss     tl_score and tl_score_backward: log probabilities, entropies and the gradient of the logits
  drop     tl_dropout: a branch added to its residual
  dropped  tl_dropout twice: the branch, and the gradient that goes back into it

Recurrence: h_t = f_t h_(t-1) + i_t x_t per channel, from a first state of each sentence; gate "sigmoid": f = sigmoid(g), i = 1 - f;
gate "given": f = g, i = 1.  Rows are all sentences' words one after the other, cut by offsets.
Scores: log softmax(x)_w, entropy of softmax(x), the `top` largest words (equal ones: lowest index first).  Gradient from those of log
probability and entropy: d_j = dl ([j = w] - p_j) - dH p_j (log p_j + H).
Dropout: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3, 2011) of the counter (column / 8, row,
step, step >> 32) under the key (seed, seed >> 32); its four words are eight pieces of 16 bits, low halves first, for eight columns side by
side.  A value whose piece is below t = round(65536 p) is dropped, others are multiplied by 65536 / (65536 - t).

listed() names twelve calls, draw() makes further ones of the same ranges, prepare() makes inputs and run() makes one call: in plain torch
operations where `own` is false, through the library's binding where it is true.  exact() evaluates the same in 64 bits, and work()
states the bytes and operations that a call cannot do without.
"""
import math

import numpy as np
import torch

own = False                 # whether run() calls the library's operators or their plain form

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases ------------------------------------------------------------------------------------------------------

def _recurrence(kind, dtype, gate, trees, lo, hi, channels, first=True, packed=False):
    """Words per sentence in [lo, hi]; first: sentences start from states of their own, not from zero; packed: gates and inputs are
    halves of one projection's rows."""
    return dict(kind=kind, dtype=dtype, gate=gate, trees=trees, lo=lo, hi=hi, channels=channels, first=first, packed=packed)


def _scores(kind, dtype, rows, vocab, top=0, entropy=True, banned=0.0, unlabelled=0.0, spread=2.5):
    """banned: share of words at -infinity; unlabelled: share of rows without a word; entropy: whether the loss depends on it;
    spread: standard deviation of the logits."""
    return dict(kind=kind, dtype=dtype, rows=rows, vocab=vocab, top=top, entropy=entropy, banned=banned, unlabelled=unlabelled, spread=spread)


def _dropout(kind, dtype, rows, cols, p, residual=True):
    return dict(kind=kind, dtype=dtype, rows=rows, cols=cols, p=p, residual=residual)


def listed():
    out = []

    def add(name, case):
        out.append(dict(case, name=name))

    # the next word of 25 sentences at the sentiment model's size: a serving step where latency counts
    add("token_sentence", _recurrence("token", "f32", "sigmoid", 25, 1, 1, 150, packed=True))
    # target sentences of a large batch, 16-bit projections
    add("scan_bulk", _recurrence("scan", "bf16", "sigmoid", 256, 5, 60, 512, packed=True))
    # two documents: one long axis, few rows beside it
    add("scan_long", _recurrence("scan", "bf16", "sigmoid", 2, 12000, 16384, 2048))
    # training steps: the paper's batch and a large batch in fp32, documents in 16 bits with gates of the caller's own
    add("train_sentence", _recurrence("train", "f32", "sigmoid", 25, 5, 60, 150, packed=True))
    add("train_bulk", _recurrence("train", "f32", "sigmoid", 256, 5, 60, 512))
    add("train_long", _recurrence("train", "bf16", "given", 8, 1500, 2048, 1024, first=False))
    # one word and its alternatives
    add("rank_one", _scores("rank", "f32", 1, 20000, top=5))
    # prompts of a batch over a wide vocabulary, with alternatives and banned words
    add("rank_wide", _scores("rank", "bf16", 512, 131072, top=20, banned=0.01))
    # losses: the paper's batch, and a large one whose loss rewards entropy and which is padded with words that do not count
    add("loss_sentence", _scores("loss", "f32", 813, 20000, entropy=False))
    add("loss_bulk", _scores("loss", "bf16", 4096, 50000, unlabelled=0.1))
    # a state's dropout in the paper's batch, and a wide one with its backward pass
    add("drop_sentence", _dropout("drop", "f32", 813, 150, 0.1))
    add("dropped_bulk", _dropout("dropped", "bf16", 65536, 1024, 0.1))
    return out


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["token", "scan", "scan", "train", "train", "train", "rank", "rank", "loss", "loss", "drop", "dropped"])
    dtype = rng.choice(["f32", "f32", "bf16", "bf16", "f16"])
    size = 4 if dtype == "f32" else 2
    if kind in ("token", "scan", "train"):
        channels = rng.choice([_log_int(rng, 1, 4096), 64 * rng.randint(1, 32), 128 * rng.randint(1, 16), rng.randint(30, 1100)])
        trees = _log_int(rng, 1, 1024)
        most = max(1, (1 << 26) // (size * channels * trees))      # words per sentence: a tensor of up to 64 MiB
        hi = 1 if kind == "token" else max(1, min(_log_int(rng, 2, 32768), most))
        lo = 1 if kind == "token" else rng.choice([0 if trees >= 4 else 1, 1, (hi + 1) // 2, hi])
        return _recurrence(kind, dtype, rng.choice(["sigmoid", "sigmoid", "given"]), trees, lo, hi, channels, rng.random() < 0.7, rng.random() < 0.5)
    if kind in ("rank", "loss"):
        vocab = _log_int(rng, 50, 131072)
        rows = max(1, min(_log_int(rng, 1, 8192), (1 << 26) // vocab))
        top = rng.choice([0, 1, rng.randint(2, 20), rng.randint(2, 64)]) if kind == "rank" else 0
        return _scores(kind, dtype, rows, vocab, min(top, vocab // 2), rng.random() < 0.5, rng.choice([0.0, 0.0, 0.02]), rng.choice([0.0, 0.1, 0.4]), rng.uniform(1.0, 4.0))
    cols = rng.choice([_log_int(rng, 1, 8192), 64 * rng.randint(1, 64), rng.randint(30, 1100)])
    rows = max(1, min(_log_int(rng, 1, 65536), (1 << 25) // cols))
    return _dropout(kind, dtype, rows, cols, rng.choice([0.1, 0.5, rng.uniform(0.0, 0.9)]), rng.random() < 0.6)


# ---- inputs -----------------------------------------------------------------------------------------------------

def _lengths(case):
    """Words of every sentence: spread over [lo, hi] in a scrambled order that the case alone fixes, so that its work does not depend on the seed."""
    i = np.arange(case["trees"])
    return (case["lo"] + np.floor(np.modf((i + 0.5) * 0.7548776662466927)[0] * (case["hi"] - case["lo"] + 1))).astype(np.int64)


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _recurrence_inputs(case, seed):
    gen, dt = _generator(seed), TYPES[case["dtype"]]
    lengths = _lengths(case)
    n, C, trees = int(lengths.sum()), case["channels"], case["trees"]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    if case["packed"]:
        both = normal(n, 2, C)
        g, x = both[:, 0], both[:, 1]
    else:
        g, x = normal(n, C), normal(n, C)
    g.mul_(1.5).add_(2.0)                                        # gates that remember for some ten words, some for hundreds
    if case["gate"] == "given":
        g.sigmoid_()
    s = dict(g=g, x=x, off=torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda(), longest=int(lengths.max()),
             h0=normal(trees, C, dtype=torch.float32) if case["first"] else None)
    if case["kind"] == "train":
        s["d_h"], s["d_last"] = normal(n, C), normal(trees, C, dtype=torch.float32)
    return s


def _score_inputs(case, seed):
    gen, n, V = _generator(seed), case["rows"], case["vocab"]
    logits = torch.randn((n, V), generator=gen, device="cuda").mul_(case["spread"])
    word = torch.randint(0, V, (n,), generator=gen, device="cuda", dtype=torch.int32)
    if case["banned"]:
        ban = torch.rand(V, generator=gen, device="cuda") < case["banned"]
        ban[word.long()] = False
        logits.masked_fill_(ban, -math.inf)
    if case["unlabelled"]:
        word[torch.rand(n, generator=gen, device="cuda") < case["unlabelled"]] = -1
    s = dict(logits=logits.to(TYPES[case["dtype"]]), word=word)
    if case["kind"] == "loss":
        scale = (1024.0 if case["dtype"] == "f16" else 1.0) / n      # (losses are scaled where gradients are fp16)
        s["d_logprob"] = torch.full((n,), -scale, device="cuda")
        s["d_entropy"] = torch.full((n,), -0.01 * scale, device="cuda") if case["entropy"] else None
    return s


def _dropout_inputs(case, seed):
    gen, dt, shape = _generator(seed), TYPES[case["dtype"]], (case["rows"], case["cols"])
    s = dict(x=torch.randn(shape, generator=gen, device="cuda", dtype=dt),
             residual=torch.randn(shape, generator=gen, device="cuda", dtype=dt) if case["residual"] else None,
             numbers=torch.randint(-2 ** 62, 2 ** 62, (2,), generator=gen, device="cuda"))          # seed and step
    if case["kind"] == "dropped":
        s["d_y"] = torch.randn(shape, generator=gen, device="cuda", dtype=dt)
    return s


def _inputs(case, seed):
    return (_recurrence_inputs if "channels" in case else _score_inputs if "vocab" in case else _dropout_inputs)(case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    torch.cuda.synchronize()
    return s


# ---- one call ---------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _own(state, case["kind"])
    return (_plain_recurrence if "channels" in case else _plain_scores if "vocab" in case else _plain_dropout)(state)


def _own(s, kind):
    from paper_1809_00832_amd import binding
    case = s["case"]
    if kind in ("token", "scan", "train"):
        gate = binding.TL_GATE_SIGMOID if case["gate"] == "sigmoid" else binding.TL_GATE_GIVEN
        out = binding.tl_recur(s["g"], s["x"], s["off"], s["h0"], gate, with_last=True, with_tape=kind == "train")
        if kind != "train":
            return out
        tape = out.pop("tape")
        return dict(out, **binding.tl_recur_backward(s["g"], s["x"], s["off"], tape, s["d_h"], s["d_last"], gate))
    if kind in ("rank", "loss"):
        out = binding.tl_score(s["logits"], s["word"], case["top"])
        answer = {k: out[k] for k in ("logprob", "entropy", "top_word", "top_logprob") if k in out}
        if kind == "loss":
            answer["d_logits"] = binding.tl_score_backward(s["logits"], s["word"], out["stats"], s["d_logprob"], s["d_entropy"])
        return answer
    y = {"y": binding.tl_dropout(s["x"], case["p"], s["numbers"], s["residual"])}
    if kind == "dropped":
        y["d_x"] = binding.tl_dropout(s["d_y"], case["p"], s["numbers"])
    return y


def _doubled(f, e, longest, back):
    """e_t + f_t (e_(t-1) + f_(t-1) (...)), or towards t + 1, for all rows at once: spans of 1, 2, 4, ... rows are joined.  f is zero where a
    sentence begins."""
    reach = 1
    while reach < longest:
        near, far = (slice(None, -reach), slice(reach, None)) if back else (slice(reach, None), slice(None, -reach))
        added, product = f[near] * e[far], f[near] * f[far]
        e[near] += added
        f[near] = product
        reach *= 2
    return e


def _plain_recurrence(s):
    """Spans of rows joined by doubling, in 32 bits."""
    case, dt, n = s["case"], s["g"].dtype, s["g"].shape[0]
    off = s["off"].long()
    begin, end = off[:-1], off[1:]
    some = begin < end                                          # (a sentence may be empty)
    first, last = begin[some], end[some] - 1
    g, x = s["g"].float(), s["x"].float()
    sigmoid = case["gate"] == "sigmoid"
    f = 1 / (1 + torch.exp(-g)) if sigmoid else g
    i = 1 / (1 + torch.exp(g)) if sigmoid else torch.ones_like(g)
    h0 = torch.zeros(case["trees"], case["channels"], device="cuda") if s["h0"] is None else s["h0"]
    e, c = i * x, f.clone()
    e[first] += f[first] * h0[some]
    c[first] = 0
    h = _doubled(c, e, s["longest"], False)
    h_last = h0.clone()
    h_last[some] = h[last]
    out = {"h": h.to(dt), "h_last": h_last}
    if case["kind"] != "train":
        return out
    before = torch.zeros_like(h)
    before[1:] = h[:-1]
    before[first] = h0[some]
    e, c = s["d_h"].to(torch.float32, copy=True), torch.zeros_like(f)
    e[last] += s["d_last"][some]
    c[:-1] = f[1:]
    c[last] = 0
    lam = _doubled(c, e, s["longest"], True)
    d_h0 = s["d_last"].clone()
    d_h0[some] = f[first] * lam[first]
    d_g = lam * (before - x) * f * i if sigmoid else lam * before
    return dict(out, d_g=d_g.to(dt), d_x=(i * lam).to(dt), d_h0=d_h0)


def _plain_scores(s):
    case = s["case"]
    x = s["logits"].float()
    n, V = x.shape
    word = s["word"].long()[:, None]
    there = (word >= 0) & (word < V)
    at = torch.where(there, word, 0)
    low = x - x.amax(dim=1, keepdim=True)
    e = torch.exp(low)
    z = e.sum(dim=1, keepdim=True)
    logp = low - torch.log(z)
    p = e / z
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(dim=1, keepdim=True)
    out = {"logprob": torch.where(there, torch.gather(logp, 1, at), 0.0)[:, 0], "entropy": entropy[:, 0]}
    if case["top"]:
        _, index = torch.sort(x, dim=1, descending=True, stable=True)          # equal ones: lowest index first
        index = index[:, :case["top"]]
        out.update(top_word=index.int(), top_logprob=torch.gather(logp, 1, index))
    if case["kind"] == "loss":
        dl = torch.where(there, s["d_logprob"][:, None], 0.0)
        d = -dl * p
        d.scatter_add_(1, at, dl)
        if s["d_entropy"] is not None:
            d -= s["d_entropy"][:, None] * torch.where(p > 0, p * (logp + entropy), 0.0)
        out["d_logits"] = d.to(s["logits"].dtype)
    return out


def _pieces(numbers, rows, cols):
    """Eight pieces of 16 bits side by side: [rows x cols]."""
    low = 0xffffffff
    k0, k1 = numbers[0] & low, (numbers[0] >> 32) & low
    blocks = (cols + 7) // 8
    c0 = torch.arange(blocks, device=numbers.device).expand(rows, blocks)
    c1 = torch.arange(rows, device=numbers.device)[:, None].expand(rows, blocks)
    c2, c3 = (numbers[1] & low).expand(rows, blocks), ((numbers[1] >> 32) & low).expand(rows, blocks)
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                 # (low 64 bits of the product, whatever their sign)
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], dim=2)
    return torch.stack([words & 0xffff, words >> 16], dim=3).view(rows, 8 * blocks)[:, :cols]


def _plain_dropout(s):
    case, dt = s["case"], s["x"].dtype
    t = int(np.rint(np.float32(case["p"]) * np.float32(65536)))
    kept = _pieces(s["numbers"], case["rows"], case["cols"]) >= t
    scale = 65536 / (65536 - t)
    y = torch.where(kept, s["x"].float() * scale, 0.0)
    out = {"y": (y if s["residual"] is None else y + s["residual"].float()).to(dt)}
    if case["kind"] == "dropped":
        out["d_x"] = torch.where(kept, s["d_y"].float() * scale, 0.0).to(dt)
    return out


# ---- what a call cannot do without ------------------------------------------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if "channels" in case:                                      # gates and inputs read, states written; training: their gradients too
        n, states = int(_lengths(case).sum()) * case["channels"], case["trees"] * case["channels"]
        train = kind == "train"
        return {"bytes": size * n * (6 if train else 3) + 4 * states * ((4 if train else 2) if case["first"] else (3 if train else 1)) + 4 * (case["trees"] + 1),
                "flops": n * (20 if train else 8)}
    if "vocab" in case:
        n = case["rows"] * case["vocab"]
        return {"bytes": size * n * (2 if kind == "loss" else 1) + 4 * case["rows"] * (3 + 2 * case["top"] + (2 if kind == "loss" else 0)),
                "flops": n * (10 if kind == "loss" else 5)}
    n = case["rows"] * case["cols"]
    return {"bytes": size * n * (2 + int(case["residual"]) + (2 if kind == "dropped" else 0)) + 16, "flops": n * 2}


# ---- the same in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    return (_exact_recurrence if "channels" in case else _exact_scores if "vocab" in case else _exact_dropout)(case, seed)


def _exact_recurrence(case, seed):
    """Word by word, all sentences side by side."""
    s = _recurrence_inputs(case, seed)
    lengths = torch.from_numpy(_lengths(case)).cuda()
    longest, trees, C = s["longest"], case["trees"], case["channels"]
    n = s["g"].shape[0]
    at = s["off"][:-1].long()
    h = torch.zeros(trees, C, dtype=torch.float64, device="cuda") if s["h0"] is None else s["h0"].double()
    before, out = torch.zeros(n, C, dtype=torch.float64, device="cuda"), torch.zeros(n, C, dtype=torch.float64, device="cuda")
    order = torch.argsort(lengths, descending=True)             # the sentences that have a t-th word are the first ones of these
    live = (lengths[order][None, :] > torch.arange(longest, device="cuda")[:, None]).sum(1).tolist()
    h, at = h[order], at[order]

    def gates(rows):
        g = s["g"][rows].double()
        return (torch.sigmoid(g), torch.sigmoid(-g)) if case["gate"] == "sigmoid" else (g, torch.ones_like(g))

    for t, m in enumerate(live):
        rows = at[:m] + t
        f, i = gates(rows)
        before[rows] = h[:m]
        h[:m] = f * h[:m] + i * s["x"][rows].double()
        out[rows] = h[:m]
    back = torch.argsort(order)
    answer = {"h": out, "h_last": h[back]}
    if case["kind"] != "train":
        return answer
    lam = s["d_last"].double()[order]
    d_g, d_x = torch.zeros_like(out), torch.zeros_like(out)
    for t in range(longest - 1, -1, -1):
        m = live[t]
        rows = at[:m] + t
        f, i = gates(rows)
        here = lam[:m] + s["d_h"][rows].double()
        d_x[rows] = here * i
        d_g[rows] = here * ((before[rows] - s["x"][rows].double()) * f * i if case["gate"] == "sigmoid" else before[rows])
        lam[:m] = here * f
    return dict(answer, d_g=d_g, d_x=d_x, d_h0=lam[back])


def _exact_scores(case, seed):
    s = _score_inputs(case, seed)
    n, V, top = case["rows"], case["vocab"], case["top"]
    parts = []
    for a in range(0, n, max(1, (1 << 25) // V)):
        b = min(n, a + max(1, (1 << 25) // V))
        x = s["logits"][a:b].double()
        logp = torch.log_softmax(x, dim=1)
        p = torch.exp(logp)
        h = -torch.xlogy(p, p).sum(1)
        word = s["word"][a:b].long()
        there = (word >= 0) & (word < V)
        rows = torch.arange(b - a, device="cuda")[there]
        l = torch.zeros(b - a, dtype=torch.float64, device="cuda")
        l[rows] = logp[rows, word[there]]
        part = {"logprob": l, "entropy": h}
        if top:
            # values in order as whole numbers, of which no two are equal once the word's number stands behind them
            bits = s["logits"][a:b].float().view(torch.int32).long()
            key = torch.where(bits < 0, -(bits & 0x7fffffff), bits) * (1 << 24) - torch.arange(V, device="cuda")
            index = torch.topk(key, top, dim=1).indices
            part.update(top_word=index.int(), top_logprob=torch.gather(logp, 1, index))
        if case["kind"] == "loss":
            d = torch.zeros_like(p)
            dl = s["d_logprob"][a:b].double() * there
            d[rows, word[there]] = dl[there]
            d -= dl[:, None] * p
            if s["d_entropy"] is not None:
                d -= s["d_entropy"][a:b].double()[:, None] * (torch.xlogy(p, p) + p * h[:, None])
            part["d_logits"] = d
        parts.append(part)
    return {k: torch.cat([q[k] for q in parts]) for k in parts[0]}


def _exact_dropout(case, seed):
    """Numbers made on the host, a part of the rows at a time."""
    s = _dropout_inputs(case, seed)
    rows, cols = case["rows"], case["cols"]
    seed_, step = (int(v) & (2 ** 64 - 1) for v in s["numbers"].tolist())
    t = round(float(np.float32(case["p"])) * 65536)
    blocks = -(-cols // 8)
    low, shift = np.uint64(0xffffffff), np.uint64(32)
    kept = np.empty((rows, cols), dtype=bool)
    for a in range(0, rows, 4096):
        b = min(rows, a + 4096)
        ctr = np.empty((4, b - a, blocks), dtype=np.uint64)
        ctr[0], ctr[1] = np.arange(blocks)[None, :], np.arange(a, b)[:, None]
        ctr[2], ctr[3] = step & 0xffffffff, step >> 32
        for r in range(10):
            key = ((seed_ + r * 0x9E3779B9) & 0xffffffff, ((seed_ >> 32) + r * 0xBB67AE85) & 0xffffffff)
            left, right = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
            ctr = np.stack([(right >> shift) ^ ctr[1] ^ np.uint64(key[0]), right & low, (left >> shift) ^ ctr[3] ^ np.uint64(key[1]), left & low])
        piece = np.ascontiguousarray(ctr.transpose(1, 2, 0).astype("<u4")).view("<u2").reshape(b - a, 8 * blocks)
        kept[a:b] = piece[:, :cols] >= t
    there = torch.from_numpy(kept).cuda()
    scale = 65536.0 / (65536 - t)
    y = s["x"].double() * there * scale
    out = {"y": y if s["residual"] is None else y + s["residual"].double()}
    if case["kind"] == "dropped":
        out["d_x"] = s["d_y"].double() * there * scale
    return out
