"""The example that writes sentences from trees: its recorded tokens against calls one by one, its gradients, a few training steps."""
import importlib.util
import os

import pytest
import torch

from paper_1809_00832_amd import binding, synth

pytestmark = pytest.mark.gpu


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


@pytest.mark.parametrize("kv_heads,leaves", [(5, False), (1, True)])
def test_replayed_tokens_are_those_of_single_calls(example, trees, kv_heads, leaves):
    w, _, batch = trees
    decoder = example.Decoder(w.params.hidden, w.params.vocab, kv_heads=kv_heads)
    mask = batch["left"] < 0 if leaves else None
    gen = torch.Generator(device="cuda").manual_seed(3)
    u = torch.rand(6, batch["B"], generator=gen, device="cuda")
    tokens, logprob = example.write(decoder, batch, 6, u, mask, top_k=40)
    k, v = (t.detach() for t in decoder.nodes(batch["h"]))
    n = batch["B"]
    one_each = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    cfg = dict(temperature=torch.full((n,), 0.8, device="cuda"), top_k=torch.full((n,), 40, dtype=torch.int32, device="cuda"),
               top_p=torch.full((n,), 0.9, device="cuda"))
    state, word = batch["h_root"], torch.zeros(n, dtype=torch.int32, device="cuda")
    with torch.no_grad():
        for i in range(6):
            x = torch.tanh(state @ decoder.w_state + decoder.words[word])
            state, logits = decoder.logits(x, lambda q: binding.tl_attend(q, k, v, one_each, batch["tree_off"], mask))
            out = binding.tl_sample(logits, u[i], **cfg)
            word = out["token"]
            assert torch.equal(tokens[i], word) and torch.equal(logprob[i], out["logprob"])
    assert int(tokens.min()) >= 0 and int(tokens.max()) < w.params.vocab


def test_gradients_through_autograd(example, trees):
    """Against autograd of the definition in 64 bits.  Sums of up to 150 products and 99 exponentials in fp32: errors stay below 300 u times the
    sums of absolute values, which the largest gradient of a tensor exceeds by far less than 30 times."""
    w, _, batch = trees
    off = batch["tree_off"].tolist()
    lq = [1 + t % 7 for t in range(batch["B"])]
    q_off = torch.tensor([0] + lq, device="cuda").cumsum(0).int()
    gen = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda").requires_grad_()
    q, k, v, g = new(sum(lq), 4, 30), new(off[-1], 2, 30), new(off[-1], 2, 30), new(sum(lq), 4, 30).detach()
    mask = batch["left"] < 0
    got = torch.autograd.grad(example.Attend.apply(q, k, v, q_off, batch["tree_off"], mask), (q, k, v), g)
    exact = [x.detach().double().cpu().requires_grad_() for x in (q, k, v)]
    Q, K, V = exact
    rows = []
    at = 0
    for t, n in enumerate(lq):
        cols = torch.arange(off[t], off[t + 1])[mask[off[t]:off[t + 1]].cpu()]
        heads = []
        for j in range(4):
            p = torch.softmax(Q[at:at + n, j] @ K[cols, j // 2].t() * 30 ** -0.5, 1)
            heads.append(p @ V[cols, j // 2])
        rows.append(torch.stack(heads, 1))
        at += n
    want = torch.autograd.grad(torch.cat(rows), exact, g.double().cpu())
    for a, b in zip(got, want):
        assert (a.double().cpu() - b).abs().max() <= 9000 * 2.0 ** -24 * b.abs().max()


def test_training_lowers_the_loss(example, trees):
    w, net, batch = trees
    decoder = example.Decoder(w.params.hidden, w.params.vocab)
    sentences, s_off = example.random_sentences(batch["B"], w.params.vocab, 5, 60, 1)
    before = batch["h"].clone()
    losses = [example.train_step(net, decoder, batch, w.params.embed_dim, sentences, s_off, 0.5).item() for _ in range(5)]
    assert all(b < a for a, b in zip(losses, losses[1:]))
    net.forward()
    assert not torch.equal(before, batch["h"])                 # the encoder has been trained too


def test_gradients_of_gradients_are_refused(example, trees):
    """Attend's backward pass is not made of differentiable steps: a second derivative raises instead of leaving out what went through it."""
    _, _, batch = trees
    n = batch["B"]
    off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(rows, 2, 16, device="cuda").requires_grad_() for rows in (n, batch["h"].shape[0], batch["h"].shape[0]))
    o = example.Attend.apply(q, k, v, off, batch["tree_off"], None)
    d_q, = torch.autograd.grad(o.square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (d_q.square().sum() + q.sum()).backward()
