"""The recurrence, dropout and the word scores together with the attention, as the example's recurrent decoder uses them; and rows far apart."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_1809_00832_amd import binding, synth
from philox import pieces

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tree_to_sentence.py")
    spec = importlib.util.spec_from_file_location("tree_to_sentence", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture()
def trees():
    w = synth.workload("sentence")
    net = binding.TreeNet(w.params, scheduler="level_device")
    batch = net.load(w.trees)
    net.forward()
    yield w, net, batch
    net.close()


def test_written_words_are_as_probable_as_scored_ones(example, trees):
    """Words drawn one by one, by replayed calls on states in place, against the same words as given sentences, in one call for all of them.  The two
    differ by the order of sums (states joined as runs; products over 150 elements): logits of size 10 to some 300 roundings, log probabilities twice that."""
    w, _, batch = trees
    decoder = example.RecurrentDecoder(w.params.hidden, w.params.vocab)
    n, B = 40, batch["B"]
    u = torch.rand(n, B, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    tokens, logprob = example.write_recurrent(decoder, batch, n, u)
    sentences = tokens.t().reshape(-1).contiguous()
    s_off = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
    got = example.score(decoder, batch, sentences, s_off, 5)
    assert (got["logprob"].view(B, n).t() - logprob).abs().max() <= 600 * U * 10
    best = got["top_logprob"]
    assert (best[:, :-1] >= best[:, 1:]).all() and (got["logprob"] <= best[:, 0]).all()
    assert (got["entropy"] > 0).all()
    alone = example.score(decoder, batch, sentences, s_off)
    assert torch.equal(alone["logprob"], got["logprob"])


def test_gradients_through_the_whole_decoder(example, trees):
    """Against autograd of the same definition in 64 bits on the host.  Sums of up to 20 000 products in fp32 behind sums of 150, and matrix products by the
    library: errors stay below 3 000 u of a tensor's largest gradient."""
    w, _, batch = trees
    H, V, B = w.params.hidden, 500, batch["B"]
    decoder = example.RecurrentDecoder(H, V, heads=5, kv_heads=1, seed=2)
    lengths = [(7 * t) % 23 for t in range(B)]                   # (the first sentence is empty)
    s_off = torch.tensor([0] + lengths, device="cuda").cumsum(0).int()
    n = sum(lengths)
    gen = torch.Generator(device="cuda").manual_seed(1)
    sentences = torch.randint(0, V, (n,), generator=gen, device="cuda", dtype=torch.int32)
    sentences[::9] = V                                          # (words that do not count)
    given = sentences.clone()
    given[::9] = 1
    numbers, p, reward = torch.tensor([77, 5], device="cuda"), 0.25, 0.1
    mask = batch["left"] < 0
    h = batch["h"].detach().clone().requires_grad_()
    root = batch["root"].long()
    k, v = decoder.nodes(h)
    state = decoder.states(example.previous_words(given, s_off), h[root], s_off)
    _, logits = decoder.logits(state, lambda q: example.Attend.apply(q, k, v, s_off, batch["tree_off"], mask), (p, numbers))
    logprob, entropy = example.LogProb.apply(logits, sentences)
    loss = -(logprob + reward * entropy).mean()
    got = torch.autograd.grad(loss, decoder.parameters() + [h])

    words, w_state, w_q, w_kv, w_o = (t.detach().double().cpu().requires_grad_() for t in decoder.parameters())
    X = h.detach().double().cpu().requires_grad_()
    last = example.previous_words(given, s_off).cpu().long()
    both = (words[last] @ w_state).view(-1, 2, H)
    kv = (X @ w_kv).view(-1, 2, 1, H // 5)
    off = batch["tree_off"].tolist()
    t_drop = int(np.rint(np.float32(p) * 65536))
    kept = torch.from_numpy(pieces(77, 5, n, H) >= t_drop).double() * (65536 / (65536 - t_drop))
    states, reads, at = [], [], 0
    for t, L in enumerate(lengths):
        s = X[root[t].cpu()]
        cols = torch.arange(off[t], off[t + 1])[mask[off[t]:off[t + 1]].cpu()]
        for r in range(at, at + L):
            f = torch.sigmoid(both[r, 0])
            s = f * s + (1 - f) * both[r, 1]
            states.append(s)
            q = (s @ w_q).view(5, -1)
            a = torch.softmax(q @ kv[cols, 0, 0].t() * (H // 5) ** -0.5, 1)
            reads.append((a @ kv[cols, 1, 0]).reshape(-1))
        at += L
    S = torch.stack(states)
    y = torch.tanh(S + kept * (torch.stack(reads) @ w_o))
    logp = torch.log_softmax(y @ words.t(), 1)
    there = (sentences < V).cpu()
    picked = torch.where(there, logp.gather(1, given.cpu().long()[:, None])[:, 0], torch.zeros(n, dtype=torch.float64))
    want_loss = -(picked - reward * (logp.exp() * logp).sum(1)).mean()
    assert abs(loss.item() - want_loss.item()) <= 1000 * U * abs(want_loss.item())
    want = torch.autograd.grad(want_loss, [words, w_state, w_q, w_kv, w_o, X])
    for a, b in zip(got, want):
        assert (a.double().cpu() - b).abs().max() <= 3000 * U * b.abs().max()


def test_training_steps_run(example, trees):
    w, net, batch = trees
    decoder = example.RecurrentDecoder(w.params.hidden, w.params.vocab)
    sentences, s_off = example.random_sentences(batch["B"], w.params.vocab, 0, 60, 1)
    numbers = torch.tensor([5, 0], device="cuda")
    before = [p.detach().clone() for p in decoder.parameters()] + [batch["h"].clone()]
    for _ in range(3):
        loss = example.recurrent_step(net, decoder, batch, w.params.embed_dim, sentences, s_off, 0.1, (0.1, numbers), 0.01)
        assert torch.isfinite(loss)
    net.forward()
    assert numbers.tolist() == [5, 3]
    assert all(not torch.equal(a, b) for a, b in zip(before, decoder.parameters() + [batch["h"]]))


def test_gradients_of_gradients_are_refused(example):
    off = torch.tensor([0, 3, 4], dtype=torch.int32, device="cuda")
    g, x, h0 = (torch.randn(n, 8, device="cuda").requires_grad_() for n in (4, 4, 2))
    d, = torch.autograd.grad(example.Recur.apply(g, x, h0, off).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (d.square().sum() + x.sum()).backward()


def test_a_training_step_is_captured_while_another_graph_of_its_leaves_lives(example):
    """Forward and backward of all three in one captured graph; the eager graph of the same leaves is gone before the recording, as torch asks."""
    B, L, C, V = 4, 9, 40, 300
    off = torch.arange(B + 1, dtype=torch.int32, device="cuda") * L
    gen = torch.Generator(device="cuda").manual_seed(0)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda")
    g, x, h0, w = new(B * L, C), new(B * L, C), new(B, C), new(C, V)
    word = torch.randint(0, V, (B * L,), generator=gen, device="cuda", dtype=torch.int32)
    numbers, dl = torch.tensor([9, 0], device="cuda"), torch.full((B * L,), -1.0 / (B * L), device="cuda")

    def step():
        out = binding.tl_recur(g, x, off, h0, with_tape=True)
        y = binding.tl_dropout(out["h"], 0.2, numbers, x)
        logits = y @ w
        s = binding.tl_score(logits, word, 3)
        d_logits = binding.tl_score_backward(logits, word, s["stats"], dl, d_logits=logits)
        d_y = d_logits @ w.t()
        back = binding.tl_recur_backward(g, x, off, out["tape"], binding.tl_dropout(d_y, 0.2, numbers))
        return [s["logprob"], s["top_word"], back["d_g"], back["d_x"] + d_y, back["d_h0"]]

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
        numbers[1:].add_(1)
    for i in range(3):
        numbers.copy_(torch.tensor([9, i], device="cuda"))
        eager = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(recorded, eager)) and numbers.tolist() == [9, i + 1]


FAR = 1_200_000_000         # elements from one row to the next: the third row begins beyond 2^31


def far(rows, cols, seed=None):
    """Rows far apart; only they are written."""
    t = torch.empty(FAR * (rows - 1) + cols, dtype=torch.bfloat16, device="cuda").as_strided((rows, cols), (FAR, 1))
    if seed is not None:
        t.copy_(torch.randn(rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
    return t


def test_rows_far_apart():
    a, b, out = far(3, 700, 1), far(3, 700, 2), far(3, 700)
    off = torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda")
    one = binding.tl_recur(a, b, off, h=out, with_last=True, with_tape=True)
    two = binding.tl_recur(a.contiguous(), b.contiguous(), off, with_last=True, with_tape=True)
    assert torch.equal(one["h"], two["h"]) and torch.equal(one["h_last"], two["h_last"])
    one = binding.tl_recur_backward(a, b, off, one["tape"], out)
    two = binding.tl_recur_backward(a.contiguous(), b.contiguous(), off, two["tape"], out.contiguous())
    assert all(torch.equal(one[k], two[k]) for k in two)
    word = torch.tensor([5, 699, 0], dtype=torch.int32, device="cuda")
    one, two = binding.tl_score(a, word, 4), binding.tl_score(a.contiguous(), word, 4)
    assert all(torch.equal(one[k], two[k]) for k in two)
    d = torch.ones(3, device="cuda")
    binding.tl_score_backward(a, word, one["stats"], d, d, d_logits=out)
    assert torch.equal(out, binding.tl_score_backward(a.contiguous(), word, one["stats"], d, d))
    numbers = torch.tensor([1, 2], device="cuda")
    binding.tl_dropout(a, 0.5, numbers, b, y=out)
    assert torch.equal(out, binding.tl_dropout(a.contiguous(), 0.5, numbers, b.contiguous()))
