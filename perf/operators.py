"""Timed cases of the operators of a decoder that writes a sentence from a tree.

The network encodes a tree bottom-up (TreeNet); a decoder then writes a sentence about it.  At every token it reads the states of
the tree's nodes by cross attention and draws a word of its vocabulary from given random numbers.

Kinds of call:
  step    tl_attend with one query per tree: the decoder's next token (serving)
  read    tl_attend with a whole target sentence per tree: scoring, or the forward half of a training step
  train   tl_attend and tl_attend_backward: outputs and the gradients of queries, keys and values
  sample  tl_sample: temperature, top-k, top-p and min-p, then one word per row from a given uniform number;
          outputs are the word, its log probability among the words kept, and their number

Queries are rows of all trees' target sentences one after the other, keys and values are rows of all trees' nodes (n = 2 L - 1
for L leaves), both cut into trees by offsets; n_heads query heads share n_kv_heads heads of keys and values.  listed() names
twelve calls, draw() makes further ones of the same ranges, prepare() makes inputs and run() makes one call: in plain torch
operations where `own` is false, through the library's binding where it is true.  exact() evaluates the same in 64 bits, and work()
states the bytes and operations that a call cannot do without.
"""
import math

import numpy as np
import torch

own = False                 # whether run() calls the library's operators or their plain form

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases ------------------------------------------------------------------------------------------------------

def _attention(kind, dtype, trees, lo, hi, q_lo, q_hi, heads, kv_heads, head_dim, mask="none", packed=False):
    """Leaves per tree in [lo, hi], target tokens per tree in [q_lo, q_hi]; mask: which nodes may be read (all; the leaves only;
    "some": a part of each tree, and nothing of every eighth tree); packed: keys and values are halves of one projection's rows."""
    return dict(kind=kind, dtype=dtype, trees=trees, lo=lo, hi=hi, q_lo=q_lo, q_hi=q_hi, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, mask=mask, packed=packed)


def _sampling(dtype, rows, vocab, temperature, top_k, top_p, min_p, mixed=False, spread=2.5):
    """0 leaves a filter out; mixed: every row has settings of its own around these; spread: standard deviation of the logits."""
    return dict(kind="sample", dtype=dtype, rows=rows, vocab=vocab, temperature=temperature, top_k=top_k, top_p=top_p,
                min_p=min_p, mixed=mixed, spread=spread)


def listed():
    out = []

    def add(name, case):
        out.append(dict(case, name=name))

    # the next token of 25 sentences, states of the sentiment model's size in five heads: a serving step where latency counts
    add("step_sentence", _attention("step", "f32", 25, 5, 50, 1, 1, 5, 5, 30))
    # the same for a large batch at the wide hidden size, query heads in groups, 16-bit states
    add("step_bulk", _attention("step", "bf16", 256, 5, 50, 1, 1, 8, 2, 64, packed=True))
    # the next token over a few documents of tens of thousands of words: one long axis, few rows
    add("step_long", _attention("step", "bf16", 4, 20000, 32768, 1, 1, 32, 8, 128))
    # scoring target sentences of a large batch
    add("read_bulk", _attention("read", "bf16", 256, 5, 50, 5, 60, 8, 8, 64, packed=True))
    # reading the leaves of large trees only, in fp32, which is what the encoder writes
    add("read_deep", _attention("read", "f32", 64, 1024, 1024, 16, 128, 4, 4, 64, mask="leaves"))
    # summaries of documents: long targets over long trees
    add("read_long", _attention("read", "bf16", 8, 1500, 2048, 512, 1024, 16, 4, 128))
    # training steps: the paper's batch and a large batch in fp32, and documents in 16 bits with nodes (and whole trees) masked
    add("train_sentence", _attention("train", "f32", 25, 5, 50, 5, 60, 5, 5, 30))
    add("train_bulk", _attention("train", "f32", 256, 5, 50, 5, 60, 8, 8, 64, packed=True))
    add("train_long", _attention("train", "bf16", 8, 700, 1024, 256, 512, 16, 4, 128, mask="some"))
    # the next word of one sentence
    add("sample_one", _sampling("f32", 1, 20000, 0.8, 0, 0.9, 0.0))
    # the next words of a large batch whose requests have settings of their own
    add("sample_batch", _sampling("f32", 256, 50000, 0.8, 50, 0.9, 0.05, mixed=True))
    # a wide vocabulary, 16-bit logits, a nucleus of many words
    add("sample_wide", _sampling("bf16", 512, 131072, 1.0, 0, 0.95, 0.0))
    return out


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step"] * 2 + ["read"] * 2 + ["train"] * 2 + ["sample"] * 2)
    if kind == "sample":
        vocab = _log_int(rng, 100, 131072)
        rows = _log_int(rng, 1, 512)
        top_k = rng.choice([0, 0, 1, _log_int(rng, 2, 1000)])
        return _sampling(rng.choice(["f32", "f32", "bf16", "f16"]), rows, vocab, rng.choice([0.0, 0.7, 1.0, 1.3, rng.uniform(0.3, 2.0)]),
                         top_k, rng.choice([0.0, 0.9, rng.uniform(0.05, 0.99)]), rng.choice([0.0, 0.0, rng.uniform(0.001, 0.3)]),
                         rng.random() < 0.4, rng.uniform(1.0, 4.0))
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    kv_heads = rng.choice([1, 2, 3, 4, 5, 8])
    group = rng.choice([1, 1, 2, 4, 7] if kv_heads < 4 else [1, 1, 2, 4])
    head_dim = rng.choice([32, 64, 64, 128, 128, _log_int(rng, 8, 256), rng.randint(1, 160)])
    if dtype == "f32" or head_dim > 128:
        group = min(group, 2)
    trees = _log_int(rng, 1, 256)
    # nodes of the batch between 64 and 32768: many short trees or few long ones
    hi = max(1, min(_log_int(rng, 2, 16384), 16384 // trees))
    lo = rng.choice([1, (hi + 1) // 2, hi])
    if kind == "step":
        q_lo, q_hi = 1, 1
    else:
        q_hi = max(1, min(_log_int(rng, 2, 1024), 8192 // trees))
        if q_hi * hi > 1 << 19:
            q_hi = max(1, (1 << 19) // hi)
        q_lo = rng.choice([0 if trees >= 4 else 1, 1, (q_hi + 1) // 2, q_hi])
    return _attention(kind, dtype, trees, lo, hi, q_lo, q_hi, kv_heads * group, kv_heads, head_dim,
                      rng.choice(["none", "none", "leaves", "some"]), rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------------------------------------------

def _spread(n, lo, hi, step):
    """n whole numbers over [lo, hi] in a scrambled order that the case alone fixes, so that its work does not depend on the seed."""
    i = np.arange(n)
    return (lo + np.floor(np.modf((i + 0.5) * step)[0] * (hi - lo + 1))).astype(np.int64)


def _lengths(case):
    """(target tokens, nodes) of every tree."""
    q = _spread(case["trees"], case["q_lo"], case["q_hi"], 0.7548776662466927)
    leaves = _spread(case["trees"], case["lo"], case["hi"], 0.6180339887498949)
    return q, 2 * leaves - 1


def _offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _mask_host(case, seed):
    """uint8 per node, or None; the leaves of a tree are as many as its case says, at places that the seed picks."""
    if case["mask"] == "none":
        return None
    rng = np.random.default_rng(seed + 1)
    _, nodes = _lengths(case)
    rows = []
    for t, n in enumerate(nodes):
        if case["mask"] == "leaves":
            row = np.zeros(n, dtype=np.uint8)
            row[rng.permutation(n)[:(n + 1) // 2]] = 1
        else:
            row = (rng.random(n) < 0.7).astype(np.uint8)
            if t % 8 == 7:
                row[:] = 0
        rows.append(row)
    return np.concatenate(rows)


def _attention_inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = TYPES[case["dtype"]]
    lq, lk = _lengths(case)
    nq, nk, D = int(lq.sum()), int(lk.sum()), case["head_dim"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dt)

    q = normal(nq, case["heads"], D)
    if case["packed"]:
        kv = normal(nk, 2, case["kv_heads"], D)
        k, v = kv[:, 0], kv[:, 1]
    else:
        k, v = normal(nk, case["kv_heads"], D), normal(nk, case["kv_heads"], D)
    mask = _mask_host(case, seed)
    s = dict(q=q, k=k, v=v, q_off=torch.from_numpy(_offsets(lq)).cuda(), kv_off=torch.from_numpy(_offsets(lk)).cuda(),
             kv_mask=None if mask is None else torch.from_numpy(mask).cuda(), scale=1.0 / math.sqrt(D),
             max_q=int(lq.max()), max_kv=int(lk.max()))
    if case["kind"] == "train":
        s["d_o"] = normal(nq, case["heads"], D)
    return s


def _settings(case, seed):
    """Per row: temperature, top_k, top_p, min_p (numpy; None where the filter is left out)."""
    rng = np.random.default_rng(seed + 2)
    n = case["rows"]

    def rows(value, lo, hi, dtype):
        if not case["mixed"]:
            return np.full(n, value, dtype=dtype)
        return np.clip(value * rng.uniform(0.5, 1.5, n), lo, hi).astype(dtype)

    out = {"temperature": rows(case["temperature"], 0.0, 4.0, np.float32), "top_k": None, "top_p": None, "min_p": None}
    if case["top_k"]:
        out["top_k"] = rows(case["top_k"], 1, case["vocab"], np.int32)
    if case["top_p"]:
        out["top_p"] = rows(case["top_p"], 0.01, 1.0, np.float32)
    if case["min_p"]:
        out["min_p"] = rows(case["min_p"], 0.0, 1.0, np.float32)
    return out


def _sampling_inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    logits = torch.randn((case["rows"], case["vocab"]), generator=gen, device="cuda").mul_(case["spread"]).to(TYPES[case["dtype"]])
    u = torch.rand(case["rows"], generator=gen, device="cuda")
    s = dict(logits=logits, u=u)
    for name, value in _settings(case, seed).items():
        s[name] = None if value is None else torch.from_numpy(value).cuda()
    return s


def prepare(case, seed):
    s = _sampling_inputs(case, seed) if case["kind"] == "sample" else _attention_inputs(case, seed)
    s["case"] = case
    torch.cuda.synchronize()
    return s


# ---- one call ---------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_1809_00832_amd import binding
        s = state
        if kind == "sample":
            return binding.tl_sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        where = dict(q_off=s["q_off"], kv_off=s["kv_off"], kv_mask=s["kv_mask"], scale=s["scale"])
        if kind != "train":
            return {"o": binding.tl_attend(s["q"], s["k"], s["v"], **where)}
        o, lse = binding.tl_attend(s["q"], s["k"], s["v"], with_lse=True, **where)
        return dict(binding.tl_attend_backward(s["q"], s["k"], s["v"], o, lse, s["d_o"], **where), o=o)
    return _plain_sample(state) if kind == "sample" else _plain_attend(state)


def _padded(off, n_max, n_rows):
    """Index of row i of every tree in the flat arrays [trees x n_max], whether there is such a row, and the tree and the place of every
    flat row."""
    at = off[:-1, None].long() + torch.arange(n_max, device=off.device)
    there = at < off[1:, None]
    rows = torch.arange(n_rows, device=off.device)
    tree = torch.bucketize(rows, off[1:].long(), right=True)
    return at.clamp(max=max(n_rows - 1, 0)), there, tree, rows - off[:-1].long()[tree]


def _plain_attend(s):
    """Trees padded to the longest, heads as batches of matrix products, in 32 bits."""
    case = s["case"]
    dt, B, Hq, Hk, D = s["q"].dtype, case["trees"], case["heads"], case["kv_heads"], case["head_dim"]
    G, Lq, Lk = Hq // Hk, s["max_q"], s["max_kv"]
    nq, nk = s["q"].shape[0], s["k"].shape[0]
    train = case["kind"] == "train"
    if nq == 0:
        out = {"o": torch.zeros_like(s["q"])}
        if train:
            out.update(d_q=torch.zeros_like(s["q"]), d_k=torch.zeros(nk, Hk, D, dtype=dt, device="cuda"),
                       d_v=torch.zeros(nk, Hk, D, dtype=dt, device="cuda"))
        return out
    q_at, q_there, q_tree, q_place = _padded(s["q_off"], Lq, nq)
    k_at, k_there, k_tree, k_place = _padded(s["kv_off"], Lk, nk)
    if s["kv_mask"] is not None:
        k_there = k_there & (s["kv_mask"] != 0)[k_at]

    def queries(x):                                            # [trees * kv heads, tokens * group, D]
        x = x.float()[q_at] * q_there[:, :, None, None]
        return x.view(B, Lq, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B * Hk, Lq * G, D)

    def nodes(x):                                              # [trees * kv heads, nodes, D], masked rows zero
        x = x.float()[k_at].masked_fill(~k_there[:, :, None, None], 0.0)
        return x.permute(0, 2, 1, 3).reshape(B * Hk, Lk, D)

    def flat_queries(x):
        x = x.view(B, Hk, Lq, G, D).permute(0, 2, 1, 3, 4)
        return x[q_tree, q_place].reshape(nq, Hq, D).to(dt)

    def flat_nodes(x):
        return x.view(B, Hk, Lk, D).permute(0, 2, 1, 3)[k_tree, k_place].to(dt)

    q, k, v = queries(s["q"]), nodes(s["k"]), nodes(s["v"])
    score = torch.bmm(q, k.transpose(1, 2).contiguous()) * s["scale"]
    live = k_there[:, None, None, :].expand(B, Hk, 1, Lk).reshape(B * Hk, 1, Lk)
    score = score.masked_fill(~live, -math.inf)
    top = score.amax(dim=2, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=2, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = torch.bmm(p, v)
    out = {"o": flat_queries(o)}
    if train:
        g = queries(s["d_o"])
        d_p = torch.bmm(g, v.transpose(1, 2).contiguous())
        d_s = p * (d_p - (g * o).sum(dim=2, keepdim=True)) * s["scale"]
        out["d_q"] = flat_queries(torch.bmm(d_s, k))
        out["d_k"] = flat_nodes(torch.bmm(d_s.transpose(1, 2).contiguous(), q))
        out["d_v"] = flat_nodes(torch.bmm(p.transpose(1, 2).contiguous(), g))
    return out


def _plain_sample(s):
    """Sorted rows, in 64 bits: which word a number picks hangs on sums over the whole vocabulary."""
    x = s["logits"].double()
    x = torch.where(torch.isnan(x), -math.inf, x)
    n, V = x.shape
    t = s["temperature"].double()[:, None]
    greedy = ~(t > 0)
    value, index = torch.sort(x, dim=1, descending=True, stable=True)     # ties: lowest index first
    rank = torch.arange(V, device=x.device)[None, :]
    w = torch.exp((value - value[:, :1]) / torch.where(greedy, 1.0, t))
    keep = ~greedy | (rank == 0)
    if s["top_k"] is not None:
        keep = keep & ((rank < s["top_k"][:, None]) | (s["top_k"][:, None] <= 0))
    w = torch.where(keep, w, 0.0)
    if s["top_p"] is not None:
        before = torch.cumsum(w, dim=1) - w
        p = s["top_p"].double()[:, None]
        keep = keep & ((before < p * w.sum(dim=1, keepdim=True)) | (rank == 0) | (p >= 1))
    if s["min_p"] is not None:
        keep = keep & (w >= s["min_p"].double()[:, None])
    w = torch.where(keep, w, 0.0)
    total = w.sum(dim=1, keepdim=True)
    by_index = torch.zeros_like(w).scatter_(1, index, w)
    run_sum = torch.cumsum(by_index, dim=1)
    token = (run_sum <= s["u"].double()[:, None] * total).sum(dim=1, keepdim=True)
    last = torch.where(by_index > 0, rank, -1).amax(dim=1, keepdim=True)
    token = torch.minimum(token, last)
    chosen = torch.gather(by_index, 1, token.clamp(min=0))
    return {"token": token[:, 0].int(), "logprob": torch.log(chosen / total)[:, 0].float(), "kept": keep.sum(dim=1).int()}


# ---- what a call cannot do without ------------------------------------------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "sample":
        settings = 1 + sum(bool(case[k]) for k in ("top_k", "top_p", "min_p"))
        n = case["rows"] * case["vocab"]
        return {"bytes": size * n + 4 * case["rows"] * (settings + 3), "flops": 2 * n}
    lq, lk = _lengths(case)
    nq, nk, pairs = int(lq.sum()), int(lk.sum()), int((lq * lk).sum())
    if case["mask"] == "leaves":
        pairs = int((lq * ((lk + 1) // 2)).sum())
    elif case["mask"] == "some":                               # seven of ten nodes, nothing of every eighth tree
        pairs = int((lq * lk * 0.7 * (np.arange(case["trees"]) % 8 != 7)).sum())
    D = case["head_dim"]
    q_bytes, kv_bytes = size * nq * case["heads"] * D, size * nk * case["kv_heads"] * D
    flops = 4 * pairs * case["heads"] * D
    bytes_ = 2 * q_bytes + 2 * kv_bytes + 8 * (case["trees"] + 1) + (nk if case["mask"] != "none" else 0)
    if case["kind"] == "train":                                # d_o read, gradients written; five products instead of two
        bytes_ += 2 * q_bytes + 2 * kv_bytes
        flops = flops * 7 // 2
    return {"bytes": bytes_, "flops": flops}


# ---- the same in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    return _exact_sample(case, seed) if case["kind"] == "sample" else _exact_attend(case, seed)


def _exact_attend(case, seed):
    """Tree by tree and head by head, from the definition."""
    s = _attention_inputs(case, seed)
    lq, lk = _lengths(case)
    mask = _mask_host(case, seed)
    G, scale = case["heads"] // case["kv_heads"], s["scale"]
    train = case["kind"] == "train"
    names = ["o", "d_q", "d_k", "d_v"] if train else ["o"]
    shape = {"o": s["q"], "d_q": s["q"], "d_k": s["k"], "d_v": s["v"]}
    out = {n: torch.zeros(tuple(shape[n].shape), dtype=torch.float64, device="cuda") for n in names}
    a = b = 0
    for tokens, nodes in zip(lq.tolist(), lk.tolist()):
        rows = slice(a, a + tokens)
        cols = np.arange(b, b + nodes)
        a, b = a + tokens, b + nodes
        if mask is not None:
            cols = cols[mask[cols] != 0]
        if tokens == 0 or len(cols) == 0:
            continue
        cols = torch.from_numpy(cols).cuda()
        K, V = s["k"][cols].double().transpose(0, 1), s["v"][cols].double().transpose(0, 1)            # [kv heads, n, D]
        for j in range(case["kv_heads"]):
            for first in range(0, tokens, 256):
                part = slice(rows.start + first, min(rows.start + first + 256, rows.stop))
                heads = slice(j * G, (j + 1) * G)
                Q = s["q"][part, heads].double()                                                        # [rows, G, D]
                P = torch.softmax(torch.matmul(Q.reshape(-1, case["head_dim"]), K[j].t()) * scale, dim=-1)
                O = torch.matmul(P, V[j])
                out["o"][part, heads] = O.view_as(Q)
                if train:
                    g = s["d_o"][part, heads].double().reshape(-1, case["head_dim"])
                    dS = P * (torch.matmul(g, V[j].t()) - (g * O).sum(-1, keepdim=True)) * scale
                    out["d_q"][part, heads] = torch.matmul(dS, K[j]).view_as(Q)
                    out["d_k"][cols, j] += torch.matmul(dS.t(), Q.reshape(-1, case["head_dim"]))
                    out["d_v"][cols, j] += torch.matmul(P.t(), g)
    return out


def _exact_sample(case, seed):
    """Row by row on the host: the least value that is kept, then the draw in the words' own order."""
    s = _sampling_inputs(case, seed)
    cfg = _settings(case, seed)
    logits, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    token = np.empty(case["rows"], dtype=np.int32)
    logprob, kept = np.empty(case["rows"]), np.ones(case["rows"], dtype=np.int32)
    for r in range(case["rows"]):
        x, t = logits[r], float(cfg["temperature"][r])
        if not t > 0:
            token[r], logprob[r] = int(np.argmax(x)), 0.0
            continue
        order = np.lexsort((np.arange(len(x)), -x))
        if cfg["top_k"] is not None and 0 < cfg["top_k"][r] < len(x):
            order = order[:cfg["top_k"][r]]
        weight = np.exp((x[order] - x[order[0]]) / t)
        if cfg["top_p"] is not None and cfg["top_p"][r] < 1:
            need = float(cfg["top_p"][r]) * weight.sum()
            n = int(np.searchsorted(np.cumsum(weight), need, side="left")) + 1        # first words that reach the mass
            order, weight = order[:n], weight[:n]
        if cfg["min_p"] is not None:
            fine = weight >= float(cfg["min_p"][r])
            order, weight = order[fine], weight[fine]
        by = np.argsort(order, kind="stable")
        order, weight = order[by], weight[by]
        kept[r] = len(order)
        total = np.cumsum(weight)
        at = min(int(np.searchsorted(total, u[r] * total[-1], side="right")), len(order) - 1)
        token[r], logprob[r] = order[at], math.log(weight[at] / total[-1])
    return {"token": torch.from_numpy(token), "logprob": torch.from_numpy(logprob), "kept": torch.from_numpy(kept)}
