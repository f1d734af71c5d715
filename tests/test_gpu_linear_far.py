"""Dense layers at the ends of their ranges: 16-bit outputs of very long sums, numbers whose squares leave fp32, gradients
that are one value for a whole row, and gradients against differences."""
import math

import pytest
import torch

from .test_gpu_linear import ACTS, HALVES, TYPES, U, act64, check, check_grad, stored

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pm(gpu_lib):
    pm = gpu_lib.ParameterManager(4, 4, 1)
    yield pm
    pm.close()


def spread(rows, columns, dtype, size=1.0):
    """Positive numbers whose sums over rows (or products of two such) are spread over the steps of a 16-bit type."""
    x = torch.rand(rows, columns, device="cuda").add_(1).mul_(0.5 * size)
    return x.mul_(torch.rand(columns, device="cuda") / 2 + 0.5).to(dtype)


# Products that the tensor cores add up for a 16-bit output before the sum is added to others in fp32.
CHAIN = {torch.float16: 8192, torch.bfloat16: 65_536}


def check_long(got, a, b):
    """got = a b, of positive numbers.  The tensor cores add 16 products at a time, each time off by two units in the last
    place (2 * 2^-23 of the sum so far) at most, all of one sign: chain / 8 * 2^-23 of the whole sum, and half of that,
    chain / 16 * 2^-23, of one that grows evenly; the chains' sums and parts of k err by half a unit each.  Then one
    rounding.  On average that rounding is off by nothing: 5 of its standard deviations (below a half step) over the root
    of the number of elements."""
    ut, _ = TYPES[got.dtype]
    k = a.shape[1]
    off = CHAIN[got.dtype] / 16 * 2.0 ** -23 + (k / CHAIN[got.dtype] + 24) * 2.0 ** -24
    for c0 in sorted({0, got.shape[1] // 128 * 64, max(0, got.shape[1] - 64)}):
        want = a.double() @ b[:, c0:c0 + 64].double()
        error = (got[:, c0:c0 + 64].double() - want) / want
        assert error.abs().max() <= off + ut * (1 + off)
        assert error.mean().abs() <= off + 5 * ut / math.sqrt(want.numel())


@pytest.mark.parametrize("rows,ins,outs", [(1 << 18, 300, 520), (1 << 18, 520, 40), (1 << 18, 24, 200), (1 << 18, 2600, 2600),
                                           (100_001, 129, 333)])
def test_long_sums_over_rows(gpu_lib, pm, rows, ins, outs):
    """dweight of many rows: tiles of every form, pairs of blocks, either order."""
    torch.manual_seed(rows + ins)
    x, g = spread(rows, ins, torch.float16, 2.0 ** -4), spread(rows, outs, torch.float16, 2.0 ** -4)
    for by_out in (False, True):
        w = stored(torch.ones(ins, outs, device="cuda", dtype=torch.float16), by_out)
        got = pm.linear_grad(x, w, g, out=gpu_lib.LinearGrads(None, torch.empty_like(w), None))
        pm.wait()
        check_long(got.weight, x.t(), g)


def test_long_sums_over_rows_bf16(gpu_lib, pm):
    torch.manual_seed(8)
    x, g = spread(1 << 20, 136, torch.bfloat16), spread(1 << 20, 328, torch.bfloat16)
    w = torch.ones(136, 328, device="cuda", dtype=torch.bfloat16)
    got = pm.linear_grad(x, w, g, out=gpu_lib.LinearGrads(None, torch.empty_like(w), None))
    pm.wait()
    check_long(got.weight, x.t(), g)


@pytest.mark.parametrize("rows", [1, 7, 64, 65, 300, 2600])
@pytest.mark.parametrize("k", [250_008, 50_021])
def test_long_sums_over_a_vocabulary(gpu_lib, pm, rows, k):
    """A product over as many words as a vocabulary has (the gradient of what its logits were made from), and the same
    with z kept, bias, activation and residual behind it; rows of 50,021 are no multiple of 16 bytes."""
    torch.manual_seed(rows)
    n = 200 if rows < 2600 else 2600
    if n == 2600 and k != 250_008:
        n = 1000
    g = spread(k, rows, torch.float16, 2.0 ** -4).t()
    if rows % 2:
        g = g.contiguous()
    w = spread(k, n, torch.float16, 2.0 ** -4)
    x = torch.ones(rows, n, device="cuda", dtype=torch.float16)
    got = pm.linear_grad(x, w.t(), g, out=gpu_lib.LinearGrads(torch.empty_like(x), None, None))
    pre, res = torch.empty(rows, n, device="cuda", dtype=torch.float16), torch.zeros(rows, n, device="cuda", dtype=torch.float16)
    out = pm.linear(g, w, torch.zeros(n, device="cuda"), "relu", res, pre=pre)
    pm.wait()
    check_long(got.x, g, w)
    check_long(pre, g, w)
    assert torch.equal(out, pre)


@pytest.mark.parametrize("act", [None, "tanh"])
@pytest.mark.parametrize("rows,ins,outs", [(9000, 256, 1000), (20_000, 1024, 1024), (65_472, 200, 328), (30_001, 333, 129)])
def test_long_sums_beside_short_ones(gpu_lib, pm, rows, ins, outs, act):
    """Both gradients of a layer, which may share a launch (dweight's sums are long, dx's are not), and the bias's."""
    torch.manual_seed(rows)
    x, g = spread(rows, ins, torch.float16, 2.0 ** -4), spread(rows, outs, torch.float16, 2.0 ** -4)
    pre = torch.randn(rows, outs, device="cuda").half() if act else None
    for by_out in (False, True):
        w = stored((torch.rand(ins, outs, device="cuda") / 8).half(), by_out)
        got, again = (pm.linear_grad(x, w, g, pre, act) for _ in range(2))
        pm.wait()
        if act is None:
            check_long(got.weight, x.t(), g)
        check_grad(x, w, g, pre, act, got)
        assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_long_sums_give_the_same_bits(gpu_lib):
    """Eager twice, and recorded in a graph and replayed twice."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        pm = gpu_lib.ParameterManager(4, 4, 1)
        x, g = torch.randn(70_000, 2600, device="cuda").half(), torch.randn(70_000, 2600, device="cuda").mul_(2.0 ** -8).half()
        w = torch.zeros(2600, 2600, device="cuda", dtype=torch.float16)
        into = [gpu_lib.LinearGrads(None, torch.empty_like(w), None) for _ in range(3)]
        for o in into[:2]:
            pm.linear_grad(x, w, g, out=o)
        pm.wait()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            pm.linear_grad(x, w, g, out=into[2])
        for _ in range(2):
            into[2].weight.zero_()
            graph.replay()
            pm.wait()
            assert torch.equal(into[2].weight, into[0].weight) and torch.equal(into[1].weight, into[0].weight)
        pm.close()


@pytest.mark.parametrize("act", ACTS)
def test_numbers_whose_squares_leave_fp32(gpu_lib, pm, act):
    """z up to 10^38, of both signs, forward and backward."""
    torch.manual_seed(3)
    z = torch.tensor([[1e18], [2e19], [1e25], [1e38], [3.0], [0.0]], device="cuda")
    z = torch.cat([z, -z]).bfloat16()
    x = torch.cat([z, torch.zeros(12, 7, device="cuda", dtype=torch.bfloat16)], 1)
    w = (torch.rand(8, 24, device="cuda") + 0.5).bfloat16()
    pre = torch.empty(12, 24, device="cuda", dtype=torch.bfloat16)
    for dtype in (torch.bfloat16, torch.float32):
        out = pm.linear(x, w, None, act, dtype=dtype, pre=pre)
        pm.wait()
        check(x, w, None, act, None, out, pre)
    grad = torch.randn(12, 24, device="cuda").bfloat16()
    into = gpu_lib.LinearGrads(torch.empty(12, 8, device="cuda"), None, torch.empty(24, device="cuda"))
    pm.linear_grad(x, w, grad, pre, act, out=into)
    pm.wait()
    check_grad(x, w, grad, pre, act, into)


@pytest.mark.parametrize("rows,ins,outs", [(6, 40, 72), (150, 136, 264), (90, 77, 131)])
def test_gradients_that_are_expanded(gpu_lib, pm, rows, ins, outs):
    """One value for a row, one row for all, one value for everything; inputs likewise."""
    torch.manual_seed(rows)
    for dtype in HALVES:
        for of in ((rows, 1), (1, outs), (1, 1)):
            grad = torch.randn(of, device="cuda").to(dtype).expand(rows, outs)
            x = torch.randn(1 if of[0] == 1 else rows, ins, device="cuda").to(dtype).expand(rows, ins)
            for by_out in (False, True):
                w = stored((torch.randn(ins, outs, device="cuda") / math.sqrt(ins)).to(dtype), by_out)
                got = pm.linear_grad(x, w, grad)
                pre = torch.randn(rows, 1, device="cuda").to(dtype).expand(rows, outs)
                curved = pm.linear_grad(x, w, grad, pre, "silu")
                pm.wait()
                check_grad(x, w, grad, None, None, got)
                check_grad(x, w, grad, pre, "silu", curved)


@pytest.mark.parametrize("act", ACTS)
def test_every_gradient_against_differences(gpu_lib, pm, act):
    """Central differences of act(z) in 64 bits at the z that the forward pass kept, times grad, through plain products.

    Differences over 2^-14: a third derivative (below 4) times 2^-28 / 6, and 2^-52 / 2^-14 of rounding.  dz is rounded to 16
    bits, a half step of each term, after a slope that is off by 32 u of grad; sums of at most 64 terms in fp32 by
    (64 / 8 + 16) 2^-23 of their magnitudes.  relu's kink lies at zero: no z is nearer to it than the difference."""
    torch.manual_seed(4)
    for dtype in HALVES:
        x, w = torch.randn(64, 24, device="cuda").to(dtype), (torch.randn(24, 40, device="cuda") / 5).to(dtype)
        b, grad = torch.randn(40, device="cuda").to(dtype), torch.randn(64, 40, device="cuda").to(dtype)
        pre = torch.empty_like(grad)
        pm.linear(x, w, b, act, pre=pre)
        pm.wait()
        pre = torch.where(pre.abs() < 2.0 ** -10, torch.full_like(pre, 2.0 ** -10), pre)
        into = gpu_lib.LinearGrads(torch.empty(64, 24, device="cuda"), torch.empty(24, 40, device="cuda"),
                                   torch.empty(40, device="cuda"))
        pm.linear_grad(x, w, grad, pre, act, out=into)
        pm.wait()
        h, z, g = 2.0 ** -14, pre.double(), grad.double()
        slope = (act64(z + h, act) - act64(z - h, act)) / (2 * h)
        dz = g * slope
        off = g.abs() * (4 * 2.0 ** -28 / 6 + 2.0 ** -37 * (1 + z.abs()) + 32 * U)
        rounded = off + (dz.abs() + off) * TYPES[dtype][0] + TYPES[dtype][1]
        more = (64 / 8 + 16) * 2.0 ** -23
        for got, left, right, of in ((into.x, dz, w.t(), 0), (into.weight, x.t(), dz, 1)):
            error = rounded @ w.double().t().abs() if of == 0 else x.double().t().abs() @ rounded
            size = left.double().abs() @ right.double().abs()
            assert ((got.double() - left.double() @ right.double()).abs() <= error + more * (size + error)).all()
        assert ((into.bias.double() - dz.sum(0)).abs() <= off.sum(0) + more * (dz.abs() + off).sum(0)).all()
