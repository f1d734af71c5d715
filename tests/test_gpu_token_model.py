"""The token-model example: its losses and trained rows against the same training in 64 bits without a parameter
manager, and that it learns in every type."""
import math

import numpy as np
import pytest
import torch

from examples import token_model as ex

pytestmark = pytest.mark.gpu


def plain(steps, vocab, dim, size, length, lr, max_norm, seed):
    """One worker's training in 64 bits: dense embedding gradients by autograd, AdaGrad on the rows that occur."""
    g = torch.Generator().manual_seed(seed)
    successors = ex.chain(vocab, g)
    theta = (torch.randn(vocab, dim, generator=g) / math.sqrt(dim)).double()
    acc = torch.full((vocab, dim), 0.1).double()
    w = [(torch.randn(*s, generator=g) / math.sqrt(s[0])).double().requires_grad_() for s in ((dim, dim), (dim, vocab))]
    data = [ex.batch(successors, size, length, g) for _ in range(steps)]
    losses = []
    for t in data:
        tokens, targets = t[:, :-1], t[:, 1:]
        table = theta.clone().requires_grad_()
        x = table[tokens] * math.sqrt(dim) * (tokens != ex.PAD).unsqueeze(-1)
        logits = torch.tanh(x @ w[0]) @ w[1]
        loss = torch.nn.functional.cross_entropy(logits.flatten(0, -2), targets.flatten(), ignore_index=ex.PAD)
        loss.backward()
        losses.append(float(loss.detach()))
        norm = math.sqrt(sum(float((q.grad ** 2).sum()) for q in (table, *w)))
        f = min(1.0, max_norm / norm)
        grad = table.grad * f
        acc += grad ** 2
        theta -= lr * grad / torch.sqrt(acc + 1e-8)
        with torch.no_grad():
            for q in w:
                q -= lr * f * q.grad
                q.grad = None
    return np.array(losses), torch.cat([theta, acc], 1).numpy()


@pytest.mark.parametrize("max_norm", [0.05, 100.0])
def test_training_equals_the_plain_one(gpu_lib, max_norm):
    """Batch losses within 1e-4 (as the fused steps' trajectories), rows within 1e-4 of the rows' scale."""
    # (products in full fp32: the dense layers are not what is compared)
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        args = dict(steps=8, vocab=300, dim=16, size=32, length=20, lr=0.1, max_norm=max_norm, seed=3)
        losses, rows = ex.train(workers=1, **args)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = before
    want, want_rows = plain(**args)
    assert np.abs(losses.numpy() - want).max() <= 1e-4 * want.max()
    assert np.abs(rows - want_rows).max() <= 1e-4 * np.abs(want_rows).max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_it_learns(gpu_lib, dtype):
    losses, _ = ex.train(steps=60, workers=2, dtype=dtype)
    first, last = losses[:4].mean(), losses[-4:].mean()
    assert torch.isfinite(losses).all() and last < 0.9 * first
