"""A next-token model whose embedding lives in the parameter manager: the token-embedding calls together.

Every worker signals the tokens of its next batch (intent), looks the rows of the current one up (embed), runs the
dense layers in PyTorch, sums the gradient rows of equal tokens (embed_grad), takes one norm over these and the dense
gradients (grad_norm), clips the dense ones in place (clip_grads), updates the embedding by AdaGrad with the same
clipping (push_grads) and advances its clock; one sync merges the clock's updates.  Nothing waits on the host: the
number of distinct tokens, the norm and the clipping factor stay on the GPU.

    python -m examples.token_model [--steps 60] [--workers 2] [--dtype bfloat16]

The data are sequences of a random chain in which every token has a few likely successors.
"""
import argparse
import math

import torch

from paper_2206_00470_gb300 import adapm

PAD = 0   # the token behind the end of a short sequence


def chain(vocab, generator, likely=4):
    """Successors of every token (token 0 is padding, and nobody's successor)."""
    return torch.randint(1, vocab, (vocab, likely), generator=generator)


def batch(successors, size, length, generator):
    """size sequences of up to length + 1 tokens, the shorter ones padded."""
    vocab, likely = successors.shape
    t = torch.empty(size, length + 1, dtype=torch.int64)
    t[:, 0] = torch.randint(1, vocab, (size,), generator=generator)
    picks = torch.randint(0, likely, (size, length), generator=generator)
    for i in range(length):
        t[:, i + 1] = successors[t[:, i], picks[:, i]]
    ends = torch.randint(length // 2 + 1, length + 2, (size, 1), generator=generator)
    return torch.where(torch.arange(length + 1) < ends, t, torch.full_like(t, PAD))


class Model:
    """Dense layers: logits = tanh(x w1) w2."""

    def __init__(self, vocab, dim, generator, dtype):
        init = lambda *shape: torch.randn(*shape, generator=generator) / math.sqrt(shape[0])   # noqa: E731
        self.params = [p.to("cuda", dtype).requires_grad_() for p in (init(dim, dim), init(dim, vocab))]

    def loss(self, x, targets):
        w1, w2 = self.params
        logits = torch.tanh(x @ w1) @ w2
        return torch.nn.functional.cross_entropy(logits.flatten(0, -2).float(), targets.flatten(), ignore_index=PAD)


def train(steps=60, workers=2, vocab=500, dim=32, size=64, length=24, lr=1.0, max_norm=4.0, dtype=torch.float32,
          seed=0):
    """The loss of every batch, and the trained embedding rows [theta | accumulators]."""
    g = torch.Generator().manual_seed(seed)
    successors = chain(vocab, g)
    rows = torch.zeros(vocab, 2 * dim)
    rows[:, :dim] = torch.randn(vocab, dim, generator=g) / math.sqrt(dim)
    rows[:, dim:] = 0.1
    model = Model(vocab, dim, g, dtype)
    pm = adapm.ParameterManager(vocab, 2 * dim, workers, init_values=rows.cuda())
    scale = math.sqrt(dim)
    # (two clocks are in hand at a time: the current batch and the one that is signalled)
    data = [[batch(successors, size, length, g).cuda() for _ in range(workers)] for _ in range(steps)]
    losses = []
    for w in range(workers):
        pm.intent(w, data[0][w][:, :-1], 0, 1)
    for clock in range(steps):
        for w in range(workers):
            if clock + 1 < steps:
                pm.intent(w, data[clock + 1][w][:, :-1], clock + 1, clock + 2)
            tokens, targets = data[clock][w][:, :-1], data[clock][w][:, 1:]
            x = pm.embed(w, tokens, dim, scale=scale, pad=PAD, dtype=dtype).requires_grad_()
            loss = model.loss(x, targets)
            loss.backward()
            dense = [p.grad for p in model.params]
            grads = pm.embed_grad(w, tokens, x.grad, scale=scale, pad=PAD)
            norm = pm.grad_norm([grads, *dense])
            pm.clip_grads(dense, norm, max_norm)
            pm.push_grads(w, grads.keys, grads.rows, lr, adagrad=True, norm=norm, max_norm=max_norm)
            with torch.no_grad():
                for p in model.params:
                    p -= lr * p.grad
                    p.grad = None
            losses.append(loss.detach())
            pm.advance_clock(w)
        pm.sync()
    pm.wait()
    rows = pm.read_main(list(range(vocab)))
    pm.close()
    return torch.stack(losses).cpu(), rows


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--dtype", choices=("float32", "bfloat16", "float16"), default="float32")
    a = ap.parse_args()
    losses, _ = train(a.steps, a.workers, dtype=getattr(torch, a.dtype))
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"batch {i:5d}  loss {float(losses[i]):.4f}")
    print(f"batch {len(losses) - 1:5d}  loss {float(losses[-1]):.4f}")


if __name__ == "__main__":
    main()
