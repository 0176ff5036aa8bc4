"""Writes a sentence from every tree of a batch, and takes training steps of the network that does.

TreeNet encodes the trees bottom-up; a one-layer decoder writes.  At every token it adds the last word's vector to its state,
reads the states of its tree's nodes by cross attention (tl_attend), and draws the next word of its vocabulary (tl_sample).  A
training step is given the sentences: one tl_attend reads for all their words, tl_attend_backward returns the gradients, and
those of the nodes' states go on through tl_backward into the encoder.  Parameters and sentences are random: there is no data set
here, and what is written means nothing.

With --recurrent the decoder's state runs along the words by a gated linear recurrence from the tree's root (tl_recur): a training step takes
whole sentences at once, with dropout (tl_dropout) and the words' log probabilities as its loss (tl_score and its gradient); a word is written by the
same calls on one row per tree, states updated in place.

    python examples/tree_to_sentence.py --tokens 20 --steps 5
    python examples/tree_to_sentence.py --recurrent
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


class Recur(torch.autograd.Function):
    """tl_recur from first states h0, with its gradients."""

    @staticmethod
    def forward(ctx, g, x, h0, off):
        out = binding.tl_recur(g, x, off, h0, with_tape=True)
        ctx.save_for_backward(g, x, off, out["tape"])
        return out["h"]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_h):
        g, x, off, tape = ctx.saved_tensors
        d = binding.tl_recur_backward(g, x, off, tape, d_h.contiguous())
        return d["d_g"], d["d_x"], d["d_h0"], None


class Dropout(torch.autograd.Function):
    """residual + dropout(x): no mask is kept, the backward pass draws the same numbers again."""

    @staticmethod
    def forward(ctx, x, residual, p, numbers):
        ctx.p = p
        ctx.save_for_backward(numbers.clone())                  # (the next step's are other ones)
        return binding.tl_dropout(x, p, numbers, residual)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_y):
        d_y = d_y.contiguous()
        return binding.tl_dropout(d_y, ctx.p, *ctx.saved_tensors), d_y, None, None


class LogProb(torch.autograd.Function):
    """Log probabilities of given words, and the entropies."""

    @staticmethod
    def forward(ctx, logits, word):
        out = binding.tl_score(logits, word)
        ctx.save_for_backward(logits, word, out["stats"])
        return out["logprob"], out["entropy"]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_logprob, d_entropy):
        return binding.tl_score_backward(*ctx.saved_tensors, d_logprob.contiguous(), d_entropy.contiguous()), None


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


class RecurrentDecoder(Decoder):
    """A decoder whose state is a gated mean of what the words so far brought, from the root of its tree on."""

    def __init__(self, hidden, vocab, **more):
        super().__init__(hidden, vocab, **more)
        self.w_state = self.w_state.detach().repeat(1, 2).requires_grad_()              # gates and inputs of the recurrence: halves of one projection's rows

    def states(self, last, h0, off):
        """State behind every word of `last` (sentences cut by off)."""
        both = (self.words[last] @ self.w_state).view(-1, 2, h0.shape[1])
        return Recur.apply(both[:, 0], both[:, 1], h0, off)

    def logits(self, h, read, drop=None):
        """drop: (share, numbers) in training."""
        o = read((h @ self.w_q).view(-1, self.heads, self.head_dim)).reshape(h.shape) @ self.w_o
        y = torch.tanh(Dropout.apply(o, h, *drop) if drop else h + o)
        return y, y @ self.words.t()


def previous_words(sentences, s_off):
    """What every word follows: a sentence's first word follows word 0."""
    last = torch.cat([sentences.new_zeros(1), sentences[:-1]])
    last[s_off[:-1][s_off[:-1] < s_off[1:]].long()] = 0
    return last


def score(decoder, batch, sentences, s_off, n_top=0, kv_mask=None):
    """tl_score of given sentences: log probability of every word, entropies, and the words that were more probable in its place."""
    with torch.no_grad():
        k, v = decoder.nodes(batch["h"])
        h = decoder.states(previous_words(sentences, s_off), batch["h_root"], s_off)
        _, logits = decoder.logits(h, lambda q: binding.tl_attend(q, k, v, s_off, batch["tree_off"], kv_mask))
        return binding.tl_score(logits, sentences, n_top)


def recurrent_loss(decoder, h, h_root, tree_off, sentences, s_off, drop=None, reward=0.0, kv_mask=None):
    """Mean of the words' negative log probabilities, less `reward` times their distributions' entropies."""
    k, v = decoder.nodes(h)
    state = decoder.states(previous_words(sentences, s_off), h_root, s_off)
    _, logits = decoder.logits(state, lambda q: Attend.apply(q, k, v, s_off, tree_off, kv_mask), drop)
    logprob, entropy = LogProb.apply(logits, sentences)
    return -(logprob + reward * entropy).mean()


def recurrent_step(net, decoder, batch, embed_dim, sentences, s_off, lr, drop=None, reward=0.0, kv_mask=None):
    """One step of gradient descent through decoder and encoder; drop: (share, numbers), whose step is counted on.  Returns the loss (a CUDA
    scalar)."""
    binding.tl_set_keep_gates(net.ctx, True)
    net.forward()
    h = batch["h"].detach().requires_grad_()
    h_root = h[batch["root"].long()]
    loss = recurrent_loss(decoder, h, h_root, batch["tree_off"], sentences, s_off, drop, reward, kv_mask)
    params = decoder.parameters()
    *grads, d_h = torch.autograd.grad(loss, params + [h])
    encoder = binding.tl_backward(net.ctx, batch, d_h.contiguous(), embed_dim)
    binding.tl_sgd_update(net.ctx, lr, batch, encoder)
    with torch.no_grad():
        for p, g in zip(params, grads):
            p.sub_(lr * g)
        if drop:
            drop[1][1:].add_(1)
    return loss.detach()


def write_recurrent(decoder, batch, n_tokens, u, kv_mask=None, temperature=1.0):
    """n_tokens words for every tree, as write does it, recorded once and replayed: the recurrence takes a row per tree and updates its states in place."""
    trees, dev = batch["B"], u.device
    hidden = batch["h_root"].shape[1]
    one_each = torch.arange(trees + 1, dtype=torch.int32, device=dev)
    warmth = torch.full((trees,), temperature, device=dev)
    state, word, number = batch["h_root"].clone(), torch.zeros(trees, dtype=torch.int32, device=dev), u[0].clone()

    @torch.no_grad()
    def token():
        both = (decoder.words[word] @ decoder.w_state).view(-1, 2, hidden)
        h = binding.tl_recur(both[:, 0], both[:, 1], one_each, state, h_last=state)["h"]
        _, logits = decoder.logits(h, lambda q: binding.tl_attend(q, k, v, one_each, batch["tree_off"], kv_mask))
        out = binding.tl_sample(logits, number, warmth)
        word.copy_(out["token"])
        return out

    with torch.no_grad():
        k, v = decoder.nodes(batch["h"])
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
    ap.add_argument("--recurrent", action="store_true", help="a state that runs along the words, dropout, the entropy's reward")
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--leaves-only", action="store_true", help="read the leaves' states alone")
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args(argv)
    w = synth.workload("sentence")
    net = binding.TreeNet(w.params, scheduler="level_device")
    batch = net.load(w.trees)
    mask = (batch["left"] < 0) if args.leaves_only else None
    decoder = (RecurrentDecoder if args.recurrent else Decoder)(w.params.hidden, w.params.vocab, seed=args.seed)
    numbers = torch.tensor([args.seed, 0], device="cuda")
    sentences, s_off = random_sentences(batch["B"], w.params.vocab, 5, 60, args.seed)
    for step in range(args.steps):
        if args.recurrent:
            loss = recurrent_step(net, decoder, batch, w.params.embed_dim, sentences, s_off, args.lr, (args.dropout, numbers), 0.01, mask)
        else:
            loss = train_step(net, decoder, batch, w.params.embed_dim, sentences, s_off, args.lr, mask)
        print("step %d: loss %.4f" % (step, loss.item()))
    net.forward()
    gen = torch.Generator(device="cuda").manual_seed(args.seed)
    u = torch.rand(args.tokens, batch["B"], generator=gen, device="cuda")
    tokens, logprob = (write_recurrent if args.recurrent else write)(decoder, batch, args.tokens, u, mask)
    if args.recurrent:
        told = score(decoder, batch, sentences, s_off, 3, mask)
        print("given sentences: log probability of a word %.2f, entropy %.2f" % (told["logprob"].mean().item(), told["entropy"].mean().item()))
    for tree in range(min(3, batch["B"])):
        print("tree %d (log probability %.2f):" % (tree, logprob[:, tree].sum().item()), *tokens[:, tree].tolist())
    net.close()


if __name__ == "__main__":
    main()
