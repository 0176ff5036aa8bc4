"""Writes a sentence from every tree of a batch, and takes training steps of the network that does.

TreeNet encodes the trees bottom-up; a one-layer decoder writes.  At every token it adds the last word's vector to its state,
reads the states of its tree's nodes by cross attention (tl_attend), and draws the next word of its vocabulary (tl_sample).  A
training step is given the sentences: one tl_attend reads for all their words, tl_attend_backward returns the gradients, and
those of the nodes' states go on through tl_backward into the encoder.  Parameters and sentences are random: there is no data set
here, and what is written means nothing.

    python examples/tree_to_sentence.py --tokens 20 --steps 5
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1809_00832_amd import binding, synth  # noqa: E402


class Attend(torch.autograd.Function):
    """tl_attend with its gradients for torch's autograd (first ones only: a second derivative raises)."""

    @staticmethod
    def forward(ctx, q, k, v, q_off, kv_off, kv_mask):
        o, lse = binding.tl_attend(q, k, v, q_off, kv_off, kv_mask, with_lse=True)
        ctx.save_for_backward(q, k, v, o, lse, q_off, kv_off, kv_mask)
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_o):
        q, k, v, o, lse, q_off, kv_off, kv_mask = ctx.saved_tensors
        g = binding.tl_attend_backward(q, k, v, o, lse, d_o.contiguous(), q_off, kv_off, kv_mask)
        return g["d_q"], g["d_k"], g["d_v"], None, None, None


class Decoder:
    """States and word vectors of the encoder's size; `heads` query heads read `kv_heads` heads of keys and values."""

    def __init__(self, hidden, vocab, heads=5, kv_heads=5, seed=0, device="cuda"):
        assert hidden % heads == 0
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, hidden // heads
        g = torch.Generator().manual_seed(seed)
        kv = 2 * kv_heads * self.head_dim

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=g) * rows ** -0.5).to(device).requires_grad_()

        self.words = (torch.randn(vocab, hidden, generator=g) * hidden ** -0.5).to(device).requires_grad_()
        self.w_state, self.w_q, self.w_kv, self.w_o = matrix(hidden, hidden), matrix(hidden, hidden), matrix(hidden, kv), matrix(hidden, hidden)

    def parameters(self):
        return [self.words, self.w_state, self.w_q, self.w_kv, self.w_o]

    def nodes(self, h):
        """Keys and values [nodes, kv_heads, head_dim] of the encoder's states: halves of one projection's rows."""
        kv = (h @ self.w_kv).view(h.shape[0], 2, self.kv_heads, self.head_dim)
        return kv[:, 0], kv[:, 1]

    def logits(self, x, read):
        """x [rows, hidden]: what the decoder knows; `read` answers queries [rows, heads, head_dim]."""
        o = read((x @ self.w_q).view(-1, self.heads, self.head_dim))
        y = torch.tanh(x + o.reshape(x.shape) @ self.w_o)
        return y, y @ self.words.t()


def write(decoder, batch, n_tokens, u, kv_mask=None, temperature=0.8, top_k=0, top_p=0.9, min_p=0.0):
    """n_tokens words for every tree: tokens [n_tokens, trees] int32 and their log probabilities.  u [n_tokens, trees]: the uniform
    numbers they are drawn with.  Every token is the same launches over the same buffers: they are recorded once and replayed."""
    trees, dev = batch["B"], u.device
    k, v = (t.detach() for t in decoder.nodes(batch["h"]))
    one_each = torch.arange(trees + 1, dtype=torch.int32, device=dev)
    full = lambda x, dt=torch.float32: torch.full((trees,), x, dtype=dt, device=dev)
    cfg = dict(temperature=full(temperature), top_k=full(top_k, torch.int32) if top_k else None, top_p=full(top_p) if top_p else None,
               min_p=full(min_p) if min_p else None)
    state, word, number = batch["h_root"].clone(), torch.zeros(trees, dtype=torch.int32, device=dev), u[0].clone()

    @torch.no_grad()
    def token():
        x = torch.tanh(state @ decoder.w_state + decoder.words[word])
        y, logits = decoder.logits(x, lambda q: binding.tl_attend(q, k, v, one_each, batch["tree_off"], kv_mask))
        state.copy_(y)
        out = binding.tl_sample(logits, number, **cfg)
        word.copy_(out["token"])
        return out

    token()                                     # (libraries set themselves up outside the recording)
    state.copy_(batch["h_root"])
    word.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = token()
    tokens = torch.empty(n_tokens, trees, dtype=torch.int32, device=dev)
    logprob = torch.empty(n_tokens, trees, device=dev)
    for i in range(n_tokens):
        number.copy_(u[i])
        graph.replay()
        tokens[i].copy_(out["token"])
        logprob[i].copy_(out["logprob"])
    return tokens, logprob


def train_step(net, decoder, batch, embed_dim, sentences, s_off, lr, kv_mask=None):
    """One step of gradient descent on the mean cross entropy of `sentences` (words of all trees' sentences one after the other, cut by
    s_off); decoder and encoder are both updated.  Returns the loss (a CUDA scalar)."""
    binding.tl_set_keep_gates(net.ctx, True)
    net.forward()
    h = batch["h"].detach().requires_grad_()
    last = torch.cat([sentences.new_zeros(1), sentences[:-1]])
    starts = s_off[:-1][s_off[:-1] < s_off[1:]].long()
    last[starts] = 0                            # a sentence's first word follows word 0
    k, v = decoder.nodes(h)
    _, logits = decoder.logits(torch.tanh(decoder.words[last]), lambda q: Attend.apply(q, k, v, s_off, batch["tree_off"], kv_mask))
    loss = torch.nn.functional.cross_entropy(logits, sentences.long())
    params = decoder.parameters()
    trained = [p for p in params if p is not decoder.w_state]           # (the state is a matter of writing only)
    *grads, d_h = torch.autograd.grad(loss, trained + [h])
    encoder = binding.tl_backward(net.ctx, batch, d_h.contiguous(), embed_dim)
    binding.tl_sgd_update(net.ctx, lr, batch, encoder)
    with torch.no_grad():
        for p, g in zip(trained, grads):
            p.sub_(lr * g)
    return loss.detach()


def random_sentences(n_trees, vocab, lo, hi, seed):
    """Stand-ins for a data set: words [n] int32 and offsets [n_trees + 1] int32."""
    rng = np.random.default_rng(seed)
    lengths = rng.integers(lo, hi + 1, n_trees)
    words = rng.integers(1, vocab, int(lengths.sum())).astype(np.int32)
    return torch.from_numpy(words).cuda(), torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=20)
    ap.add_argument("--steps", type=int, default=5, help="training steps before the sentences are written")
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--leaves-only", action="store_true", help="read the leaves' states alone")
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args(argv)
    w = synth.workload("sentence")
    net = binding.TreeNet(w.params, scheduler="level_device")
    batch = net.load(w.trees)
    mask = (batch["left"] < 0) if args.leaves_only else None
    decoder = Decoder(w.params.hidden, w.params.vocab, seed=args.seed)
    sentences, s_off = random_sentences(batch["B"], w.params.vocab, 5, 60, args.seed)
    for step in range(args.steps):
        loss = train_step(net, decoder, batch, w.params.embed_dim, sentences, s_off, args.lr, mask)
        print("step %d: loss %.4f" % (step, loss.item()))
    net.forward()
    gen = torch.Generator(device="cuda").manual_seed(args.seed)
    u = torch.rand(args.tokens, batch["B"], generator=gen, device="cuda")
    tokens, logprob = write(decoder, batch, args.tokens, u, mask)
    for tree in range(min(3, batch["B"])):
        print("tree %d (log probability %.2f):" % (tree, logprob[:, tree].sum().item()), *tokens[:, tree].tolist())
    net.close()


if __name__ == "__main__":
    main()
