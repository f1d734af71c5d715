"""The token model with its dense layers in the library: the gradients of a step against the same step in 64 bits, all
calls of a step together in a recorded graph against the same calls made one by one, and that the example runs.

Tolerance of the gradients: nine values on the way are rounded to 11 bits (x, h, pre, u, logits, their gradient, and those
of u, z and h), each off by at most 2^-11 of itself, and no step multiplies what came before by more than 3 in norm here:
32 * 2^-11 of a gradient's norm."""
import math

import numpy as np
import pytest
import torch

from examples import token_model as ex

pytestmark = pytest.mark.gpu


def step64(x, params, ids, targets):
    """Loss and gradients by autograd on the formulas."""
    leaves = [x.double().requires_grad_(), *(p.double().requires_grad_() for p in params)]
    e, gain, shift, w1, b1, w2 = leaves
    m = e.mean(-1, keepdim=True)
    h = (e - m) / torch.sqrt(((e - m) ** 2).mean(-1, keepdim=True) + 1e-5) * gain + shift
    logits = (torch.tanh(h @ w1 + b1) + e) @ w2
    T = ex.ManagerModel.temperature
    log_q, log_c = torch.log_softmax(logits / T, -1), torch.log_softmax(logits, -1)
    likely = ids.shape[-1]
    kl = (-math.log(likely) - log_q.gather(-1, ids)).mean(-1)
    ce = -log_c.gather(-1, targets.unsqueeze(-1)).squeeze(-1)
    known = targets != ex.PAD
    loss = (torch.where(known, ex.ManagerModel.soft * T * T * kl + ex.ManagerModel.hard * ce, 0.0) / known.sum()).sum()
    loss.backward()
    return float(loss.detach()), [t.grad for t in leaves]


@pytest.mark.parametrize("vocab,dim,size,length", [(300, 32, 16, 20), (1001, 65, 5, 33), (20_000, 128, 4, 11)])
def test_gradients_of_a_step(gpu_lib, vocab, dim, size, length):
    g = torch.Generator().manual_seed(vocab)
    successors = ex.chain(vocab, g)
    model = ex.ManagerModel(vocab, dim, g, torch.float16)
    data = ex.batch(successors, size, length, g).cuda()
    tokens, targets = data[:, :-1], data[:, 1:]
    ids = successors.cuda()[tokens]
    x = torch.randn(size, length, dim, generator=g).cuda().half()
    pm = gpu_lib.ParameterManager(4, 4, 1)
    loss, dx, dense = model.step(pm, x, ids, targets)
    pm.wait()
    want, grads = step64(x, model.params, ids, targets)
    assert abs(float(loss) - want) <= 32 * 2.0 ** -11 * abs(want)
    for got, t in zip([dx, *dense], grads):
        assert torch.linalg.vector_norm(got.double() - t) <= 32 * 2.0 ** -11 * torch.linalg.vector_norm(t)
    # padded positions have no gradient
    assert not dx[targets == ex.PAD].any()
    pm.close()


def test_a_whole_step_in_a_graph(gpu_lib):
    """From the lookup to the update: launches of a recorded step against the same calls one by one, bit for bit."""
    vocab, dim, size, length = 700, 48, 6, 15
    g = torch.Generator().manual_seed(5)
    successors = ex.chain(vocab, g)
    rows = torch.cat([torch.randn(vocab, dim, generator=g) / 7, torch.full((vocab, dim), 0.1)], 1).cuda()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        likely = successors.cuda()
        pair = [gpu_lib.ParameterManager(vocab, 2 * dim, 1, init_values=rows) for _ in range(2)]
        models = [ex.ManagerModel(vocab, dim, torch.Generator().manual_seed(1), torch.bfloat16) for _ in pair]
        data = ex.batch(successors, size, length, g).cuda()
        tokens, targets = data[:, :-1], data[:, 1:]

        def step(pm, model):
            x = pm.embed(0, tokens, dim, scale=3.0, pad=ex.PAD, dtype=torch.bfloat16)
            loss, dx, dense = model.step(pm, x, likely[tokens], targets)
            grads = pm.embed_grad(0, tokens, dx, scale=3.0, pad=ex.PAD)
            norm = pm.grad_norm([grads, *dense])
            pm.clip_grads(dense, norm, 0.5)
            pm.push_grads(0, grads.keys, grads.rows, 0.1, adagrad=True, norm=norm, max_norm=0.5)
            for p, d in zip(model.params, dense):
                p -= 0.1 * d
            return loss

        for pm, model in zip(pair, models):
            step(pm, model)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            recorded = step(pair[0], models[0])
        for _ in range(3):
            data.copy_(ex.batch(successors, size, length, g))
            graph.replay()
            eager = step(pair[1], models[1])
            for pm in pair:
                pm.wait()
            assert torch.equal(recorded, eager)
            keys = np.arange(vocab)
            assert np.array_equal(pair[0].read_main(keys), pair[1].read_main(keys))
            for a, b in zip(models[0].params, models[1].params):
                assert torch.equal(a, b)
        for pm in pair:
            pm.close()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_the_example_runs(gpu_lib, dtype):
    losses, rows = ex.train(steps=12, workers=2, dtype=dtype, layers="manager")
    assert losses.shape == (24,) and torch.isfinite(losses).all() and np.isfinite(rows).all()
