"""Trains a small byte-level language model around the gated linear recurrence, then writes with it token by token.

    python examples/train_recurrence.py [--steps 60] [--width 256] [--bits 8]

A block is a dense projection to q, k, v and g, featurizer convolutions on q, k, v, the recurrence, and a dense projection
back, as a residual.  The loss is the cross entropy of the hidden states against the embedding's rows, its gradients come from
the library, and so does the optimiser.  The text is made here: sentences of a tiny grammar, packed into one row, each of which
resets the memory at its first byte.
"""
import argparse
import math
import os
import random
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2503_01868_amd as hy  # noqa: E402

VOCABULARY = 256
GROUP = 16          # channels that share a decay
TAPS = 4            # of the featurizers


class Featurize(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, h):
        ctx.save_for_backward(x, h)
        return hy.hyena_featurize_fwd(x, h)

    @staticmethod
    def backward(ctx, dy):
        x, h = ctx.saved_tensors
        return hy.hyena_featurize_bwd(dy.contiguous(), x, h)


class Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, g):
        y, _, marks = hy.hyena_glr_fwd_carry(q, k, v, g, GROUP, want_state=False, want_marks=True)
        ctx.save_for_backward(q, k, v, g, marks)
        return y

    @staticmethod
    def backward(ctx, dy):
        q, k, v, g, marks = ctx.saved_tensors
        return hy.hyena_glr_bwd(dy, q, k, v, g, GROUP, marks=marks)[:4]


class CrossEntropy(torch.autograd.Function):
    """The mean loss of the rows that have a target."""

    @staticmethod
    def forward(ctx, x, w, target):
        loss, lse = hy.hyena_xent_fwd(x, w, target)
        weight = ((target >= 0) & (target < w.shape[0])).float()
        weight /= weight.sum()
        ctx.save_for_backward(x, w, target, lse, weight)
        return (loss * weight).sum()

    @staticmethod
    def backward(ctx, d):
        x, w, target, lse, weight = ctx.saved_tensors
        dx, dw = hy.hyena_xent_bwd(weight * d, x, w, target, lse)
        return dx, dw, None


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Model:
    def __init__(self, width, blocks, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def param(*shape, scale, dtype=torch.bfloat16):
            p = (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)
            return p.requires_grad_()

        self.width = width
        self.embedding = param(VOCABULARY, width, scale=1 / math.sqrt(width))
        self.blocks = []
        for _ in range(blocks):
            into = param(3 * width + width // GROUP, width, scale=1 / math.sqrt(width))
            taps = [param(width, TAPS, scale=1 / math.sqrt(TAPS), dtype=torch.float32) for _ in range(3)]
            self.blocks.append((into, taps, param(width, width, scale=0.5 / math.sqrt(width))))

    def parameters(self):
        return [self.embedding] + [p for into, taps, out in self.blocks for p in (into, *taps, out)]

    def gates(self, fused, first):
        """q, k, v and the log decay of every step; a document's first step forgets."""
        q, k, v, r = fused.split([self.width] * 3 + [self.width // GROUP], -1)
        g = -torch.nn.functional.softplus(-4 - r.float())  # time constants around 50 steps
        if first is not None:
            g = torch.where(first[..., None], -math.inf, g)
        return q, k, v, g.to(q.dtype)

    def hidden(self, tokens, first):
        x = self.embedding[tokens] * math.sqrt(self.width)
        for into, taps, out in self.blocks:
            q, k, v, g = self.gates(norm(x) @ into.t(), first)
            q, k, v = (Featurize.apply(t.contiguous(), h) for t, h in zip((q, k, v), taps))
            x = x + Recurrence.apply(q, k, v, g) @ out.t()
        return norm(x)

    def loss(self, tokens, first):
        x = self.hidden(tokens, first)[:, :-1]
        target = tokens[:, 1:].masked_fill(first[:, 1:], -1)  # the first byte of a document is not to be foreseen
        return CrossEntropy.apply(x.reshape(-1, self.width), self.embedding, target.reshape(-1))

    @torch.no_grad()
    def write(self, prompt, count):
        """The likeliest bytes behind `prompt`, one at a time, to the end of the sentence: per block a state and the featurizers'
        last inputs."""
        states = [torch.zeros(1, self.width, device="cuda") for _ in self.blocks]
        pasts = [torch.zeros(3, TAPS, self.width, device="cuda") for _ in self.blocks]
        text = list(prompt)
        for i in range(len(prompt) + count - 1):
            x = self.embedding[text[i]][None] * math.sqrt(self.width)
            for state, past, (into, taps, out) in zip(states, pasts, self.blocks):
                q, k, v, g = self.gates(norm(x) @ into.t(), None)
                past.copy_(torch.roll(past, 1, 1))
                past[:, 0] = torch.stack([q[0], k[0], v[0]]).float()
                q, k, v = (((past[j] * taps[j].t()).sum(0)[None]).to(x.dtype) for j in range(3))
                x = x + hy.hyena_glr_step(q, k, v, g.contiguous(), state, GROUP) @ out.t()
            if i + 1 == len(text):
                text.append(int((norm(x) @ self.embedding.t()).argmax()))
                if text[-1] == ord("\n"):
                    break
        return bytes(text)


def documents(rng, length):
    """`length` bytes of sentences, and where each begins."""
    text, first = bytearray(), []
    while len(text) < length:
        sentence = "the %s %s the %s.\n" % (rng.choice(["cat", "dog", "crow"]), rng.choice(["sees", "hears", "follows"]),
                                            rng.choice(["river", "moon", "old road"]))
        first.append(len(text))
        text += sentence.encode()
    return text[:length], [f for f in first if f < length]


def batch(rng, rows, length):
    tokens, first = torch.zeros(rows, length, dtype=torch.int64), torch.zeros(rows, length, dtype=torch.bool)
    for r in range(rows):
        text, begins = documents(rng, length)
        tokens[r] = torch.tensor(list(text))
        first[r, begins] = True
    return tokens.cuda(), first.cuda()


def train(steps=60, width=256, blocks=2, rows=8, length=256, bits=8, seed=0, say=print):
    """(losses, model) of a short training run."""
    model, rng = Model(width, blocks, seed), random.Random(seed)
    # dense weights in bf16 with fp32 masters; the filters are fp32 and do not decay
    groups = []
    for dtype, decay in ((torch.bfloat16, 0.1), (torch.float32, 0.0)):
        params = [p for p in model.parameters() if p.dtype == dtype]
        for p in params:
            p.grad = torch.zeros_like(p)  # in place from here on: the optimiser's table holds their addresses
        state = hy.adamw_state(params, bits, masters=dtype == torch.bfloat16)
        groups.append(hy.plan_adamw([p.detach() for p in params], [p.grad for p in params], weight_decay=decay, **state))
    losses = []
    for step in range(1, steps + 1):
        loss = model.loss(*batch(rng, rows, length))
        for p in model.parameters():
            p.grad.zero_()
        loss.backward()
        size = torch.sqrt(sum(p.grad.float().square().sum() for p in model.parameters()))
        clip = (1.0 / size.clamp(min=1.0)).reshape(1)
        for plan in groups:
            plan(lr=3e-3, step=step, grad_scale=clip)
        losses.append(float(loss.detach()))
        if step % 10 == 0 or step == 1:
            say("step %d: loss %.3f" % (step, losses[-1]))
    return losses, model


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=60)
    parser.add_argument("--width", type=int, default=256)
    parser.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = parser.parse_args()
    _, trained = train(a.steps, a.width, bits=a.bits)
    print(trained.write(b"the cat", 40).decode("ascii", "replace"))
