"""Distillation of rows far from zero, at temperatures far from one, and of rows whose parts hold nothing: against the
formula in 64 bits.

Tolerances (u = 2^-24).  As in test_gpu_distill.py an exponential errs by 4 u of itself and 3 u D, D at most 88 where it
counts in fp32 (e^-88 is the smallest normal number), 268 u, and its sum by 64 u (4000 u for rows read twice).  A factor
that is part of the exponent adds 2^-17, 128 u.  Together 460 u (4460 u) of each term of a gradient, then one rounding
to its type; a loss errs by as much times the magnitudes of its terms and one for the logarithms of the sums.  An
exponential below 2^-126 counts as 0.  Sums are at least 1 (the largest logit's term), so a probability loses 2^-126 at
most by that, and a gradient, of two of each kind, 2 (soft T + hard) 2^-126 scale: 10^-34 for a scale of 4096, which bf16
holds."""
import math

import pytest
import torch

from .test_gpu_distill import TYPES, U, lists, wanted

pytestmark = pytest.mark.gpu

HALVES = [torch.float16, torch.bfloat16]
# rows, vocabulary: one launch for all (short and long rows); a row in a block's registers, two and eight words a thread;
# slices of one block and of a cluster's; read twice
SHAPES = [(5, 1000), (5, 30_000), (200, 1000), (200, 5000), (200, 20_001), (200, 50_000), (3, 530_000)]


@pytest.fixture(scope="module")
def pm(gpu_lib):
    pm = gpu_lib.ParameterManager(4, 4, 1)
    yield pm
    pm.close()


def check(pm, logits, ids, teacher, T, soft=1.0, labels=None, hard=0.0, scale=1.0):
    n, V = logits.shape
    weights = torch.rand(n, device="cuda") / 2 + 0.5
    loss, size, grad, gsize = wanted(logits, ids, teacher, T, soft, labels, hard, None, scale, weights)
    into = torch.full_like(logits, 3.0)
    got = pm.distill(logits, ids, teacher, T, soft, labels, hard, scale=scale, weights=weights, grad=into)
    pm.wait()
    k = 4460 if V * logits.element_size() > 1_000_000 else 460
    assert ((got.double() - loss).abs() <= k * U * (size + 1.0 + abs(soft) * T * T + abs(hard))).all()
    ut, tiny = TYPES[logits.dtype]
    gone = 2 * (abs(soft) * T + abs(hard)) * scale * 2.0 ** -126
    assert ((into.double() - grad).abs() <= k * U * gsize + grad.abs() * ut + tiny + gone).all()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("n,V", SHAPES)
def test_a_factor_in_the_exponent(gpu_lib, pm, n, V, dtype):
    """Rows of a few neighbouring numbers of the type, from near zero to the largest: the softmax has many terms."""
    torch.manual_seed(n + V)
    for base, T in ((40.0, 1.0), (100.0, 1.0), (60.0, 0.01), (1000.0, 1.0), (-3000.0, 1.0), (10_000.0, 3.0), (-40_000.0, 10.0),
                    (60_000.0, 1.0)):
        step = torch.finfo(dtype).eps * 2.0 ** math.floor(math.log2(abs(base)))
        logits = (base + step * torch.randint(0, 7, (n, V), device="cuda")).to(dtype)
        ids, teacher = lists((n,), V, 9)
        check(pm, logits, ids, teacher, T, scale=4096.0)
        check(pm, logits, None, None, 1.0, labels=ids[:, 0].contiguous(), hard=1.0, scale=4096.0)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("n,V", SHAPES)
def test_temperatures_far_from_one(gpu_lib, pm, n, V, dtype):
    """Differences that one temperature needs where the other one, or the plain exponential, sees nothing but the largest."""
    torch.manual_seed(n + V + 1)
    ids, teacher = lists((n,), V, 9)
    labels = ids[:, 2].contiguous()
    near = (torch.randn(n, V, device="cuda") * 2).to(dtype)
    for T in (1e-5, 3e-6):
        check(pm, near, ids, teacher, T, 1.0, labels, 1.0, scale=4096.0)
    far = (torch.rand(n, V, device="cuda") * (100_000 if dtype is torch.bfloat16 else 60_000)).to(dtype)
    for T in (4000.0, 30_000.0):
        check(pm, far, ids, teacher * 1000, T, 1.0, None, 0.0, scale=1 / 16)
        check(pm, far, ids, teacher * 1000, T, 1.0, labels, 1.0, scale=1 / 16)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,V", SHAPES)
def test_no_number_among_masked_words(gpu_lib, pm, n, V, dtype):
    """A NaN whose part of the row holds nothing but -infinity beside it makes the row NaN, and no other row; parts of
    -infinity alone, or of rows of nothing else, do as they did."""
    torch.manual_seed(n + V + 2)
    logits = torch.randn(n, V, device="cuda").to(dtype)
    ids, teacher = lists((n,), 90, 5)
    logits[:3, 100:] = -math.inf
    logits[0, V - 1] = math.nan
    logits[1, V // 2:] = math.nan
    if n > 4:
        logits[3] = -math.inf
        logits[4] = math.nan
    bad = [0, 1] + ([3, 4] if n > 4 else [])
    good = [i for i in range(n) if i not in bad]
    for T, labels, hard in ((1.0, None, 0.0), (2.0, ids[:, 0].contiguous(), 0.5), (0.7, ids[:, 0].contiguous(), 0.5)):
        into = torch.zeros_like(logits)
        loss = pm.distill(logits, ids, teacher, T, 1.0, labels, hard, grad=into)
        pm.wait()
        assert loss[bad].isnan().all() and into[bad].isnan().all()
        assert torch.isfinite(loss[good]).all() and torch.isfinite(into[good]).all()
