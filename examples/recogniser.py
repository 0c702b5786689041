"""A small recogniser, trained and then run as a stream.

    python examples/recogniser.py [--steps 40] [--utterances 8]

Frames of random utterances over a random lexicon go through a gated
recurrence; a linear layer turns its states into the weights of emission graphs
(one arc a token), which are composed with the lexicon.  The loss of an
utterance is the lexicon's score of all token strings minus the score of the one
that was said (0 when no other word string is likely); a second head learns which
word ends at a frame by cross entropy over the whole vocabulary.  The gradients
go back from the arcs of the composed graphs to the emissions, the recurrence
and the layers.  Then frames arrive one at a time, and the recurrence's single
steps give the states of the whole sequence.

The network's own products (x = frames w) are torch's; everything between them
and the loss is this library's.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2110_02848_amd import gpu, synth  # noqa: E402

F32 = torch.float32


def utterances(rng, n, spellings, tokens, width, noise=1.0):
    """n utterances of 3 to 6 words: their tokens and, at each frame, the word
    that ends there (-1: none); frames are noisy embeddings of the tokens."""
    embed = rng.standard_normal((tokens, width)).astype(np.float32)
    out = []
    for _ in range(n):
        words = rng.integers(0, len(spellings), rng.integers(3, 7))
        tok = np.concatenate([spellings[w] for w in words]) - 1
        ends = np.full(len(tok), -1, np.int32)
        ends[np.cumsum([len(spellings[w]) for w in words]) - 1] = words
        frames = embed[tok] + noise * rng.standard_normal((len(tok), width)).astype(np.float32)
        out.append((tok, ends, frames))
    return out


class Recogniser:
    def __init__(self, comp, lexicon, tokens, words, width, hidden, dtype=torch.bfloat16, seed=0):
        self.comp, self.lexicon, self.tokens, self.dtype = comp, lexicon, tokens, dtype
        g = torch.Generator(device="cuda").manual_seed(seed)

        def layer(rows, cols):  # kept in float32, used in dtype
            return torch.randn(rows, cols, generator=g, device="cuda") / cols ** 0.5
        self.layers = dict(x=layer(hidden, width), gate=layer(hidden, width),
                           token=layer(tokens, hidden), word=layer(words, hidden))

    def used(self):
        return {k: v.to(self.dtype) for k, v in self.layers.items()}

    def loss_and_grads(self, batch):
        """(lattice loss, word loss) per frame, and gradients of the layers."""
        comp, w = self.comp, self.used()
        lens = [len(tok) for tok, _, _ in batch]
        bounds = np.concatenate([[0], np.cumsum(lens)])
        offset = torch.tensor(bounds, dtype=torch.int32, device="cuda")
        N = int(bounds[-1])
        frames = torch.from_numpy(np.concatenate([f for _, _, f in batch])).cuda().to(self.dtype)
        said = torch.from_numpy(np.concatenate([t for t, _, _ in batch])).cuda().long()
        ends = torch.from_numpy(np.concatenate([e for _, e, _ in batch])).cuda()

        x, gate = frames @ w["x"].t(), frames @ w["gate"].t()
        rec = comp.recurrence(x, gate, offset, save=True)
        h = rec["y"]

        # emissions of all utterances, composed with the lexicon in one pass
        weight = comp.emission_weights(h, w["token"])
        graphs = [self._emissions(weight[bounds[i]:bounds[i + 1]]) for i in range(len(batch))]
        C, states, arcs = comp.compose_batch(graphs, self.lexicon, keys=False)
        sc = comp.score(C)
        totals = comp.segment_logsum(sc["alpha"], C["accept"], states)
        post = comp.posterior(C, sc["alpha"], sc["beta"], sc["total"])
        # posteriors within each utterance, not within the batch
        share = torch.repeat_interleave(torch.exp(sc["total"] - totals),
                                        torch.from_numpy(np.diff(arcs)).cuda())
        post = (post.double() * share).float() / N
        grad = comp.grad_scatter(post, C["arc_a"], N * self.tokens).view(N, self.tokens)
        path = torch.gather(weight, 1, said[:, None])
        grad.scatter_add_(1, said[:, None], torch.full_like(path, -1.0 / N))
        lattice = (totals.sum() - path.double().sum()) / N

        words = comp.cross_entropy(h, w["word"], ends)
        some = int((ends >= 0).sum())
        coef = torch.full((N,), 1.0 / some, device="cuda")

        gh, g_token = comp.emission_grads(h, w["token"], weight, grad)
        gh2, g_word = comp.cross_entropy_grads(h, w["word"], ends, words["lse"], coef)
        back = comp.recurrence_grads(x, gate, offset, gh + gh2, rec["saved"])
        grads = dict(x=back["x"].t() @ frames, gate=back["gate"].t() @ frames, token=g_token,
                     word=g_word)
        return float(lattice), float(words["loss"].sum() / some), grads

    def _emissions(self, weight):
        """The emission graph of one utterance: state t has an arc to t + 1 for
        every token, its weights the rows of `weight` as they lie."""
        T, C = weight.shape
        i32 = dict(dtype=torch.int32, device="cuda")
        src = torch.arange(T, **i32).repeat_interleave(C)
        label = torch.arange(1, C + 1, **i32).repeat(T)
        flags = torch.zeros(2, T + 1, dtype=torch.uint8, device="cuda")
        flags[0, 0] = flags[1, T] = 1
        off = torch.clamp(torch.arange(T + 2, **i32), max=T) * C
        return dict(num_states=T + 1, arc_offset=off, src=src, dst=src + 1, ilabel=label,
                    olabel=label, weight=weight.reshape(-1), start=flags[0], accept=flags[1])

    def step(self, grads, rate):
        for k, g in grads.items():
            self.layers[k] -= rate * g.to(F32)

    def stream(self, frames):
        """States of frames that arrive one at a time."""
        w = self.used()
        state = torch.zeros(1, self.layers["x"].shape[0], device="cuda")
        out = []
        for f in frames:
            f = f[None]
            y, state = self.comp.recurrence_step(f @ w["x"].t(), f @ w["gate"].t(), state)
            out.append(y)
        return torch.cat(out)


def main(steps=40, n=8, words=200, tokens=24, width=40, hidden=128, rate=1.0, seed=0,
         dtype=torch.bfloat16):
    """Trains for `steps` steps on fresh utterances; returns the losses of each
    step and how far the stream's states are from the sequence's."""
    rng = np.random.default_rng(seed)
    comp = gpu.Composer(0)
    graph, spellings = synth.lexicon(rng, words, tokens, 2, 6)
    net = Recogniser(comp, gpu.to_device(graph), tokens, words, width, hidden, dtype, seed)
    data = utterances(rng, n * 8, spellings, tokens, width)
    losses = []
    for k in range(steps):
        batch = [data[i] for i in rng.choice(len(data), n, replace=False)]
        lattice, word, grads = net.loss_and_grads(batch)
        net.step(grads, rate)
        losses.append((lattice, word))
        print(f"step {k}: lattice loss {lattice:.4f} a frame, word loss {word:.3f}", flush=True)
    frames = torch.from_numpy(data[0][2]).cuda().to(dtype)
    w = net.used()
    whole = comp.recurrence(frames @ w["x"].t(), frames @ w["gate"].t(),
                            torch.tensor([0, len(frames)], dtype=torch.int32, device="cuda"))["y"]
    apart = float((net.stream(frames).float() - whole.float()).abs().max())
    print(f"stream and sequence apart by at most {apart:.3g}", flush=True)
    comp.close()
    return losses, apart


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--utterances", type=int, default=8)
    args = ap.parse_args()
    main(args.steps, args.utterances)
