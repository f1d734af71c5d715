"""Distillation from a teacher's top logits against the formula in 64 bits.

Tolerances (u = 2^-24).  With D the distance of a logit from its row's largest in units of the temperature, an
exponential errs by 4 u of itself (its function) and 3 u D (difference, product, argument); D is at most 64 wherever the
exponential counts in fp32 sums of these inputs, so every probability errs by 200 u of itself, its sum (eight to 64
numbers one after the other, then trees; 4,000 for rows read twice) by 64 u or 4000 u more.  A gradient errs by that of
each of its terms, then one rounding to its type.  A loss errs by 300 u (or 4000 u) times the magnitudes of its terms
and one for the logarithms of the sums."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {torch.float32: (2.0 ** -24, 2.0 ** -126), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -126)}
DTYPES = list(TYPES)


@pytest.fixture(scope="module")
def pm(gpu_lib):
    pm = gpu_lib.ParameterManager(4, 4, 1)
    yield pm
    pm.close()


def wanted(logits, ids, teacher, T, soft, labels, hard, pad, scale, weights):
    """Losses and gradients in 64 bits, and the magnitudes of what they are sums of."""
    V = logits.shape[-1]
    s = logits.reshape(-1, V).double()
    n = s.shape[0]
    loss, size = (torch.zeros(n, dtype=torch.float64, device=s.device) for _ in range(2))
    grad, gsize = torch.zeros_like(s), torch.zeros_like(s)
    f = torch.full((n, 1), float(torch.tensor(scale, dtype=torch.float32)), dtype=torch.float64, device=s.device)
    if weights is not None:
        f = f * weights.reshape(n, 1).double()
    if ids is not None and soft != 0:
        i, t = ids.reshape(n, -1).long(), teacher.reshape(n, -1).double()
        here = (i >= 0) & (i < V) & (t != -math.inf)
        some = here.any(-1, keepdim=True)
        p = torch.where(some, torch.softmax((t / T).masked_fill(~here, -math.inf), -1), 0.0)
        lq = torch.log_softmax(s / T, -1)
        at = i.clamp(0, V - 1)
        lp = torch.log_softmax((t / T).masked_fill(~here, -math.inf), -1)
        terms = torch.where(p > 0, p * (lp - lq.gather(-1, at)), torch.zeros_like(p))
        loss += soft * T * T * terms.sum(-1)
        size += abs(soft) * T * T * torch.where(p > 0, p * (lp.abs() + lq.gather(-1, at).abs()), torch.zeros_like(p)).sum(-1)
        q = torch.where(some, lq.exp(), 0.0)
        dense = torch.zeros_like(s).scatter_add_(-1, at, torch.where(here, p, torch.zeros_like(p)))
        grad += soft * T * (q - dense)
        gsize += abs(soft) * T * (q + dense)
    if labels is not None and hard != 0:
        y = labels.reshape(n, 1).long()
        marked = (y >= 0) & (y < V) if pad is None else (y >= 0) & (y < V) & (y != pad)
        lc = torch.log_softmax(s, -1)
        one = torch.zeros_like(s).scatter_(-1, y.clamp(0, V - 1), 1.0)
        loss += torch.where(marked.squeeze(-1), -hard * lc.gather(-1, y.clamp(0, V - 1)).squeeze(-1), 0.0)
        size += torch.where(marked.squeeze(-1), abs(hard) * lc.gather(-1, y.clamp(0, V - 1)).squeeze(-1).abs(), 0.0)
        grad += torch.where(marked, hard * (lc.exp() - one), 0.0)
        gsize += torch.where(marked, abs(hard) * (lc.exp() + one), 0.0)
    return loss, size, grad * f, gsize * f.abs()


def check(pm, logits, ids=None, teacher=None, T=1.0, soft=1.0, labels=None, hard=0.0, pad=None, scale=1.0, weights=None,
          in_place=False, long=False):
    kept = logits.clone() if in_place else None
    loss, size, grad, gsize = wanted(logits, ids, teacher, T, soft, labels, hard, pad, scale, weights)
    into = logits if in_place else torch.full(logits.shape, 3.0, dtype=logits.dtype, device="cuda")
    args = dict(ids=ids, teacher=teacher, temperature=T, soft=soft, labels=labels, hard=hard, pad=pad, scale=scale,
                weights=weights)
    alone = pm.distill(logits, **args)
    got = pm.distill(logits, grad=into, **args)
    pm.wait()
    assert got.shape == logits.shape[:-1]
    k = 4300 if long else 300
    hardness = 1.0 + abs(soft) * T * T + abs(hard)
    for t in (got, alone):
        assert ((t.reshape(-1).double() - loss).abs() <= k * U * (size + hardness)).all()
    ut, tiny = TYPES[logits.dtype]
    off = (into.reshape(grad.shape).double() - grad).abs()
    assert (off <= k * U * gsize + grad.abs() * ut + tiny).all()
    if in_place:
        logits.copy_(kept)
    return got, into


def lists(lead, V, top, id_type=torch.int64, dtype=torch.float32):
    at = torch.rand((*lead, V), device="cuda").argsort(-1)[..., :top] if V <= 4096 else \
        (torch.randint(1, max(2, V // top), (*lead, top), device="cuda").cumsum(-1)
         + torch.randint(0, V, (*lead, 1), device="cuda")) % V
    return at.to(id_type), (torch.randn((*lead, top), device="cuda") * 2 + 3).to(dtype)


# one element to rows over a cluster of sixteen blocks, and longer; around the limits of every kernel
VOCABS = [1, 2, 5, 8, 50, 127, 1000, 2040, 2048, 2049, 4096, 8176, 8184, 8185, 16_376, 16_380, 32_003, 50_021, 65_537, 131_072,
          250_000, 300_001, 524_281, 530_000, 700_000]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", VOCABS)
def test_every_vocabulary(gpu_lib, pm, V, dtype):
    torch.manual_seed(V)
    for n in (1, 5 if V > 100_000 else 37):
        logits = (torch.randn(n, V, device="cuda") * 2).to(dtype)
        ids, teacher = lists((n,), V, min(V, 20), torch.int32 if V % 2 else torch.int64, dtype)
        long = V * logits.element_size() > 1_000_000
        check(pm, logits, ids, teacher, long=long)
        labels = torch.randint(0, V, (n,), device="cuda")
        labels[::2] = ids[::2, 0].long()
        check(pm, logits, ids, teacher, 2.0, 0.7, labels, 0.3, scale=256.0 / n, long=long)
        check(pm, logits, labels=labels, hard=1.0, in_place=True, long=long)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [3, 100, 3001, 20_001, 100_003])
def test_rows_that_begin_anywhere(gpu_lib, pm, V, dtype):
    """Logits and gradients that begin on every element of a 16-byte word, each on its own."""
    n = 4
    buf = torch.randn(n * (V + 3) + 32, device="cuda").to(dtype)
    ids, teacher = lists((n,), V, min(V, 9))
    labels = torch.randint(0, V, (n,), device="cuda")
    for a in range(0, 9):
        logits = buf[a:a + n * (V + 3)].view(n, V + 3)[:, :V]
        want = None
        for b in (a, 0, 1, 3, 6):
            dst = torch.full((n * (V + 5) + 32,), 3.0, dtype=dtype, device="cuda")
            into = dst[b:b + n * (V + 5)].view(n, V + 5)[:, :V]
            loss = pm.distill(logits, ids, teacher, 1.5, 0.6, labels, 0.4, grad=into)
            pm.wait()
            if want is None:
                want = wanted(logits, ids, teacher, 1.5, 0.6, labels, 0.4, None, 1.0, None)
            # (sums are taken word by word of the gradient's row: their order, not their bound, goes by where it begins)
            l64, size, grad, gsize = want
            assert ((loss.double() - l64).abs() <= 300 * U * (size + 3)).all()
            ut, tiny = TYPES[dtype]
            assert ((into.double() - grad).abs() <= 300 * U * gsize + grad.abs() * ut + tiny).all()
            again = into.clone()
            pm.distill(logits, ids, teacher, 1.5, 0.6, labels, 0.4, grad=into)
            pm.wait()
            assert torch.equal(into, again)
            # what lies in front, between and behind stays
            mask = torch.ones_like(dst, dtype=torch.bool)
            mask[b:b + n * (V + 5)].view(n, V + 5)[:, :V] = False
            assert (dst[mask] == 3.0).all()


@pytest.mark.parametrize("V", [40, 3000, 32_003])
def test_few_rows_equal_many(gpu_lib, pm, V):
    """One launch does at most as many rows as there are SMs, three do more: losses and gradients of the same rows."""
    n = 400
    for dtype, T in ((torch.bfloat16, 1.0), (torch.float32, 2.0), (torch.float16, 3.0)):
        logits = (torch.randn(n, V, device="cuda") * 2).to(dtype)
        ids, teacher = lists((n,), V, min(V, 17))
        labels = torch.randint(0, V, (n,), device="cuda")
        labels[5:9], ids[7:12] = -100, -1
        check(pm, logits, ids, teacher, T, 0.5, labels, 0.5, pad=-100)
        for a in (0, 150, 300):
            check(pm, logits[a:a + 100], ids[a:a + 100], teacher[a:a + 100], T, 0.5, labels[a:a + 100], 0.5, pad=-100)
            check(pm, logits[a:a + 100], ids[a:a + 100], teacher[a:a + 100], T, in_place=True)


def test_strides_and_types(gpu_lib, pm):
    B, T, V = 3, 10, 501
    wide = torch.randn(B, T + 1, V, device="cuda")
    ids, teacher = lists((B, T), V, 7, torch.int32, torch.bfloat16)
    labels = torch.randint(0, V, (B, T + 1), device="cuda")
    check(pm, wide[:, :-1], ids, teacher, 0.7, 1.0, labels[:, 1:], 0.5)
    check(pm, wide[:, :-1].transpose(0, 1), ids.transpose(0, 1), teacher.transpose(0, 1))
    check(pm, wide[0, 0], ids[0, 0], teacher[0, 0])
    check(pm, wide[:, :-1], ids, teacher.half(), weights=torch.rand(B, T, device="cuda"), scale=-3.0)
    # one list for all rows, one row of logits for all lists
    check(pm, wide[:, :-1], ids[:1, :1].expand(B, T, 7), teacher[:1, :1].expand(B, T, 7))
    check(pm, wide[:1, :1].expand(B, T, V), ids, teacher)


@pytest.mark.parametrize("V", [64, 5000, 40_000])
def test_rows_with_little_to_learn_from(gpu_lib, pm, V):
    """Shorter lists, lists of nothing, padded labels, neither: loss 0 and zeros, whatever the logits hold."""
    n = 24
    logits = torch.randn(n, V, device="cuda").to(torch.bfloat16)
    ids, teacher = lists((n,), V, 6)
    labels = torch.randint(0, V, (n,), device="cuda", dtype=torch.int32)
    ids[0:4, 2:] = -1
    ids[4:8] = -1
    teacher[8:12] = -math.inf
    teacher[12:14, :3] = -math.inf
    labels[2:6] = -100
    labels[10] = -100
    check(pm, logits, ids, teacher, 2.0, 0.5, labels, 0.5, pad=-100)
    check(pm, logits, ids, teacher, 1.0, 0.5, labels, 0.5, pad=2 ** 32 - 100)   # the same label in 32 bits
    logits[4], logits[10] = math.nan, math.inf
    into = torch.full_like(logits, 5.0)
    loss = pm.distill(logits, ids, teacher, 2.0, 0.5, labels, 0.5, pad=-100, grad=into)
    pm.wait()
    for r in (4, 5, 10):
        assert loss[r] == 0 and not into[r].any()
    assert torch.isfinite(loss).all()
    # nothing at all
    into.fill_(5.0)
    loss = pm.distill(logits, grad=into)
    pm.wait()
    assert not loss.any() and not into.any()
    # with soft or hard 0 the other one alone counts
    check(pm, logits[11:], ids[11:], teacher[11:], 3.0, 0.0, labels[11:], 2.0)
    check(pm, logits[11:], ids[11:], teacher[11:], 3.0, 1.0, labels[11:], 0.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_words_of_the_vocabulary(gpu_lib, pm, dtype):
    """Logits of -infinity and of the type's lowest value, rows of nothing else, and what is no number."""
    n, V = 10, 9000
    logits = torch.randn(n, V, device="cuda").to(dtype)
    ids, teacher = lists((n,), V, 5)
    logits[0:3, 100:8000] = -math.inf
    logits[3:6, 100:8000] = torch.finfo(dtype).min
    logits[6] = torch.finfo(dtype).min          # all the same: uniform
    ids[:] = torch.tensor([1, 5, 99, 8000, 8999], device="cuda")
    check(pm, logits[:8], ids[:8], teacher[:8], 2.0, 1.0, ids[:8, 1].contiguous(), 1.0)
    # an entry whose logit is masked: an infinite loss, a finite gradient
    ids[0, 2] = 500
    into = torch.empty_like(logits)
    logits[8] = -math.inf
    logits[9, 17] = math.nan
    loss = pm.distill(logits, ids, teacher, grad=into)
    pm.wait()
    assert loss[0] == math.inf and torch.isfinite(into[0]).all() and into[0, 500] < 0
    assert loss[8:].isnan().all() and into[8:].isnan().all() and torch.isfinite(loss[1:8]).all()


@pytest.mark.parametrize("top", [2, 33, 256, 1024])
@pytest.mark.parametrize("V", [30, 3000, 70_000])
def test_ids_listed_twice(gpu_lib, pm, V, top):
    torch.manual_seed(top)
    n = 9
    logits = torch.randn(n, V, device="cuda")
    ids = torch.randint(0, V, (n, top), device="cuda")
    ids[0] = 7 % V
    ids[1, ::2] = 3
    teacher = torch.randn(n, top, device="cuda")
    teacher[2, ::3] = -math.inf
    labels = ids[:, top // 2].clone()
    got, grad = check(pm, logits, ids, teacher, 1.3, 1.0, labels, 1.0)
    again = torch.empty_like(grad)
    for _ in range(3):
        pm.distill(logits, ids, teacher, 1.3, 1.0, labels, 1.0, grad=again)
        pm.wait()
        assert torch.equal(again, grad)


def test_far_logits(gpu_lib, pm):
    """Entries of probability zero, and a student that is sure."""
    logits = torch.randn(6, 3000, device="cuda")
    ids, teacher = lists((6,), 3000, 8)
    teacher[:, 0] = 500.0
    logits[3, 17] = 300.0
    check(pm, logits, ids, teacher, 0.5)
    teacher[:] = 1e30
    check(pm, logits, ids, teacher, 1.0)
    logits[2] = 1e30
    logits[2, 5] = 2e30
    loss = pm.distill(logits, ids, teacher)
    pm.wait()
    assert not loss.isnan().any()


def test_logits_far_from_zero(gpu_lib, pm):
    """An offset of all logits of a row changes nothing but their own rounding."""
    for V in (300, 20_000, 300_001):
        logits = torch.randn(4, V, device="cuda") * 2 + torch.tensor([[1000.0], [-3000.0], [30.0], [20_000.0]], device="cuda")
        ids, teacher = lists((4,), V, 8)
        check(pm, logits, ids, teacher, 1.0, long=V > 270_000)
        check(pm, logits, ids, teacher, 1.7, 0.5, ids[:, 0].contiguous(), 0.5, long=V > 270_000)


def test_ids_outside_the_vocabulary_are_reported(gpu_lib):
    pm = gpu_lib.ParameterManager(4, 4, 1)
    V = 50
    logits = torch.randn(4, V, device="cuda")
    ids, teacher = lists((4,), V, 5)
    labels = torch.tensor([1, 2, 3, 4], device="cuda")
    for where, value in ((ids, V), (ids, -2), (ids, 2 ** 40), (labels, V), (labels, -1)):
        keep = where.clone()
        where[(0, 1) if where.dim() == 2 else 1] = value
        loss, into = torch.empty(4, device="cuda"), torch.empty_like(logits)
        pm.distill(logits, ids, teacher, 1.0, 1.0, labels, 1.0, grad=into, loss=loss)
        with pytest.raises(gpu_lib.AdaPMError) as e:
            pm.wait()
        assert e.value.status == gpu_lib.ERANGE
        l64, size, grad, gsize = wanted(logits, ids, teacher, 1.0, 1.0, labels, 1.0, None, 1.0, None)
        assert ((loss.double() - l64).abs() <= 300 * U * (size + 3)).all()
        assert ((into.double() - grad).abs() <= 300 * U * gsize + U * grad.abs() + 2.0 ** -126).all()
        where.copy_(keep)
    pm.distill(logits, ids, teacher)
    pm.wait()
    pm.close()


def test_gradient_against_differences(gpu_lib, pm):
    torch.manual_seed(2)
    logits = torch.randn(2, 40, device="cuda")
    ids, teacher = lists((2,), 40, 6)
    labels = torch.tensor([3, 5], device="cuda")
    grad = torch.empty_like(logits)
    pm.distill(logits, ids, teacher, 1.7, 0.4, labels, 0.6, grad=grad)
    pm.wait()
    f = lambda x: wanted(x, ids, teacher, 1.7, 0.4, labels, 0.6, None, 1.0, None)[0].sum()   # noqa: E731
    for at in ((0, 3), (0, int(ids[0, 0])), (1, 39), (1, int(ids[1, 2]))):
        up, down = logits.double().clone(), logits.double().clone()
        up[at] += 1e-5
        down[at] -= 1e-5
        slope = float(f(up) - f(down)) / 2e-5
        # (differences: 1e-10 of third derivatives and 1e-11 of rounding; the gradient: 300 u of its terms)
        assert abs(float(grad[at]) - slope) <= 300 * U * 2 + 1e-9


def test_recorded_in_a_graph(gpu_lib):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        pm = gpu_lib.ParameterManager(4, 4, 1)
        for V in (700, 90_000):
            logits = torch.randn(6, V, device="cuda")
            ids, teacher = lists((6,), V, 12)
            grad, loss = torch.empty_like(logits), torch.empty(6, device="cuda")
            pm.distill(logits, ids, teacher, grad=grad, loss=loss)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                pm.distill(logits, ids, teacher, grad=grad, loss=loss)
            for _ in range(3):
                logits.copy_(torch.randn(6, V, device="cuda"))
                teacher.copy_(torch.randn(6, 12, device="cuda"))
                g.replay()
                got = loss.clone(), grad.clone()
                pm.distill(logits, ids, teacher, grad=grad, loss=loss)
                torch.cuda.synchronize()
                assert torch.equal(got[0], loss) and torch.equal(got[1], grad)
        pm.close()


def test_refusals(gpu_lib, pm):
    x = torch.zeros(4, 8, device="cuda")
    ids, t = torch.zeros(4, 3, device="cuda", dtype=torch.int64), torch.zeros(4, 3, device="cuda")
    y = torch.zeros(4, device="cuda", dtype=torch.int64)
    flat = torch.zeros(100, device="cuda")
    big = torch.zeros(4, 1025, device="cuda")
    bad = [
        lambda: pm.distill(x.cpu(), ids, t),
        lambda: pm.distill(x.double(), ids, t),
        lambda: pm.distill(x, ids),
        lambda: pm.distill(x, None, t),
        lambda: pm.distill(x, ids[:, :2], t),
        lambda: pm.distill(x, ids[:3], t[:3]),
        lambda: pm.distill(x, ids.float(), t),
        lambda: pm.distill(x, ids.cpu(), t),
        lambda: pm.distill(x, ids, t.cpu()),
        lambda: pm.distill(x, big.long(), big),
        lambda: pm.distill(x, ids, t, 0.0),
        lambda: pm.distill(x, ids, t, -1.0),
        lambda: pm.distill(x, ids, t, 1e-39),
        lambda: pm.distill(x, ids, t, math.nan),
        lambda: pm.distill(x, ids, t, math.inf),
        lambda: pm.distill(x, ids, t, soft=math.nan),
        lambda: pm.distill(x, labels=y[:3], hard=1.0),
        lambda: pm.distill(x, labels=y.short(), hard=1.0),
        lambda: pm.distill(x, ids, t, weights=torch.zeros(3, device="cuda")),
        lambda: pm.distill(x, ids, t, loss=torch.zeros(3, device="cuda")),
        lambda: pm.distill(x, ids, t, loss=torch.zeros(4, device="cuda").half()),
        lambda: pm.distill(x, ids, t, grad=x.half()),
        lambda: pm.distill(x, ids, t, grad=torch.zeros(4, 9, device="cuda")),
        lambda: pm.distill(x, ids, t, grad=flat.as_strided((4, 8), (4, 1))),
        lambda: pm.distill(flat.as_strided((4, 8), (9, 1)), ids, t, grad=flat.as_strided((4, 8), (8, 1))),
        lambda: pm.distill(torch.zeros(4, 0, device="cuda"), ids, t),
        lambda: pm.distill(x, ids, t, weights=flat[:4], loss=flat[:4]),
        lambda: pm.distill(x, ids, t, weights=flat[:4], grad=flat.as_strided((4, 8), (8, 1))),
        lambda: pm.distill(t, ids, t, grad=t),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, gpu_lib.AdaPMError)) as e:
            call()
        assert not isinstance(e.value, gpu_lib.AdaPMError) or e.value.status == gpu_lib.EINVAL, i
    pm.wait()
    assert not flat.any()
    assert pm.distill(torch.zeros(0, 8, device="cuda"), ids[:0], t[:0]).shape == (0,)


def test_offsets_beyond_32_bits(gpu_lib, pm):
    """More than 2^31 logits: the rows behind that are like the others."""
    n, V = 8700, 250_000
    logits = torch.empty(n, V, dtype=torch.bfloat16, device="cuda")
    for a in range(0, n, 300):
        logits[a:a + 300].normal_(0.0, 2.0)
    ids, teacher = lists((n,), V, 4)
    part = [0, 1, 8600, 8698, 8699]
    kept = logits[part].clone()
    loss = pm.distill(logits, ids, teacher, grad=logits)
    pm.wait()
    l64, size, grad, gsize = wanted(kept, ids[part], teacher[part], 1.0, 1.0, None, 0.0, None, 1.0, None)
    assert ((loss[part].double() - l64).abs() <= 300 * U * (size + 2)).all()
    ut, tiny = TYPES[torch.bfloat16]
    assert ((logits[part].double() - grad).abs() <= 300 * U * gsize + grad.abs() * ut + tiny).all()
    # what the softmax's parts sum to: 1 - 1, but for their roundings
    assert (logits[8000:].double().sum(1).abs() <= 2.0 ** -8 * 2).all()
