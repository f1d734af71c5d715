"""Layer norm and its gradient against the formulas in 64 bits.

Tolerances (u = 2^-24).  A sum over a row of `dim` elements adds at most depth = max(32, dim / 1024 + 16) numbers one
after the other (eight of a lane, then trees; a strided loop for long rows).  With A = mean |x| and r the reciprocal
deviation, the mean errs by depth u A, a difference from it by that and u of itself, the deviation by 2 depth u (1 + A r)
of itself: h errs by depth u (4 |h| (1 + A r) + A r).  The gradients' sums over a row err by depth u of the sums of
magnitudes, their sums over n rows by (n / 152 + 300) u of those (the rows of a block one after the other, at most 256
groups of it, at most 8 * 152 * 4 blocks in eight strands of trees).  Then one rounding to the output's type."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {torch.float32: (2.0 ** -24, 2.0 ** -149), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}
DTYPES = list(TYPES)
DIMS = [1, 2, 7, 8, 9, 31, 64, 100, 200, 255, 256, 257, 300, 333, 1001, 1024, 2050, 4096, 8184, 8192, 8193, 20_000, 40_003]


@pytest.fixture(scope="module")
def pm(gpu_lib):
    pm = gpu_lib.ParameterManager(4, 4, 1)
    yield pm
    pm.close()


def depth(dim):
    return max(32, dim // 1024 + 16)


def forward64(x, w, b, eps):
    x = x.double()
    m = x.mean(-1, keepdim=True)
    r = ((x - m).square().mean(-1, keepdim=True) + eps).rsqrt()
    h = (x - m) * r
    y = h
    if w is not None:
        y = y * w.double()
    if b is not None:
        y = y + b.double()
    return m, r, h, y


def check_forward(x, w, b, eps, out, stats=None):
    m, r, h, y = forward64(x, w, b, eps)
    dim = x.shape[-1]
    a = x.double().abs().mean(-1, keepdim=True) * r
    err = depth(dim) * U * (4 * h.abs() * (1 + a) + a)
    if w is not None:
        err = err * w.double().abs()
    err = err + 3 * U * (y.abs() + (b.double().abs() if b is not None else 0))
    ut, tiny = TYPES[out.dtype]
    assert ((out.double() - y).abs() <= err * (1 + ut) + y.abs() * ut + tiny).all()
    if stats is not None:
        s = stats.double()
        assert ((s[..., 0:1] - m).abs() <= depth(dim) * U * x.double().abs().mean(-1, keepdim=True) + 2.0 ** -149).all()
        assert ((s[..., 1:2] - r).abs() <= depth(dim) * U * 2 * r * (1 + a)).all()


def check_grad(x, grad, stats, w, got):
    n, dim = x.numel() // x.shape[-1], x.shape[-1]
    m, r = stats.double().unsqueeze(-2).unbind(-1)
    h = (x.double() - m) * r
    dy = grad.double()
    g = dy * w.double() if w is not None else dy
    if got.x is not None:
        want = r * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
        size = r.abs() * (g.abs() + g.abs().mean(-1, keepdim=True) + h.abs() * (g * h).abs().mean(-1, keepdim=True))
        ut, tiny = TYPES[got.x.dtype]
        assert ((got.x.double() - want).abs() <= (depth(dim) + 8) * U * size + want.abs() * ut + tiny).all()
    for t, terms in ((got.weight, dy * h), (got.bias, dy)):
        if t is None:
            continue
        terms = terms.reshape(n, dim)
        want, ut, tiny = terms.sum(0), *TYPES[t.dtype]
        assert ((t.double() - want).abs() <= (n / 152 + 300) * U * terms.abs().sum(0) + want.abs() * ut + tiny).all()


def rows(shape, dtype, mean=0.3, std=1.5):
    return (torch.randn(shape, device="cuda") * std + mean).to(dtype)


def params(dim, dtype):
    return (torch.randn(dim, device="cuda") * 0.2 + 1).to(dtype), (torch.randn(dim, device="cuda") * 0.2).to(dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_every_width(gpu_lib, pm, dim, dtype):
    torch.manual_seed(dim)
    for n in (1, 3, 700 if dim < 5000 else 9):
        x = rows((n, dim), dtype)
        w, b = params(dim, torch.float32 if dim % 2 else dtype)
        stats = torch.empty(n, 2, device="cuda")
        out = pm.layer_norm(x, w, b, eps=1e-5, stats=stats)
        pm.wait()
        check_forward(x, w, b, 1e-5, out, stats)
        grad = rows((n, dim), dtype, 0.0, 0.1)
        got = pm.layer_norm_grad(x, grad, stats, w)
        pm.wait()
        assert got.x.dtype == dtype and got.weight.dtype == got.bias.dtype == w.dtype
        check_grad(x, grad, stats, w, got)


@pytest.mark.parametrize("x_type", DTYPES)
@pytest.mark.parametrize("y_type", DTYPES)
@pytest.mark.parametrize("dim", [64, 1000, 9000])
def test_types_of_their_own(gpu_lib, pm, x_type, y_type, dim):
    x, n = rows((33, dim), x_type), 33
    for p in DTYPES:
        w, b = params(dim, p)
        stats = torch.empty(n, 2, device="cuda")
        out = pm.layer_norm(x, w, b, dtype=y_type, stats=stats)
        pm.wait()
        assert out.dtype == y_type
        check_forward(x, w, b, 1e-5, out, stats)
        got = pm.layer_norm_grad(x, out, stats, w)
        pm.wait()
        check_grad(x, out, stats, w, got)


VIEWS = [
    lambda d: torch.randn(5, 12, d, device="cuda")[:, :-1],            # all but the last position
    lambda d: torch.randn(12, 5, d, device="cuda").transpose(0, 1),    # positions first
    lambda d: torch.randn(40, d + 5, device="cuda")[:, 3:d + 3],       # columns of a wider buffer
    lambda d: torch.randn(40, 2 * d, device="cuda")[::2, :d],
    lambda d: torch.randn(d, device="cuda"),                           # one row
    lambda d: torch.randn(2, 3, 4, 5, d, device="cuda")[:, 1:, :, ::2],   # more than two steps: copied
    lambda d: torch.randn(d, 11, device="cuda").t(),                   # elements apart: copied
    lambda d: torch.randn(1, d, device="cuda").expand(9, d),           # one row nine times
]


@pytest.mark.parametrize("view", range(len(VIEWS)))
@pytest.mark.parametrize("dim", [24, 133, 512, 8200])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides(gpu_lib, pm, view, dim, dtype):
    x = VIEWS[view](dim)
    if dtype is not torch.float32:   # (the view's own strides in another type)
        size = 1 + sum((n - 1) * s for n, s in zip(x.shape, x.stride()))
        flat = torch.as_strided(x, (size,), (1,)).to(dtype)
        x = torch.as_strided(flat, x.shape, x.stride())
    w, b = params(dim, torch.float32)
    stats = torch.empty(*x.shape[:-1], 2, device="cuda")
    out = pm.layer_norm(x, w, b, stats=stats)
    pm.wait()
    check_forward(x, w, b, 1e-5, out, stats)
    # an output of other strides, whose neighbours stay
    wide = torch.full((*x.shape[:-1], dim + 16), 7.0, device="cuda", dtype=dtype)
    if x.dim() <= 3:
        pm.layer_norm(x, w, b, out=wide[..., 8:dim + 8])
        pm.wait()
        assert torch.equal(wide[..., 8:dim + 8], out) and (wide[..., :8] == 7).all() and (wide[..., dim + 8:] == 7).all()
    grad = torch.randn(x.shape, device="cuda").to(dtype)
    got = pm.layer_norm_grad(x, grad, stats, w)
    pm.wait()
    check_grad(x, grad, stats, w, got)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [65, 97, 333, 1023, 1025, 4001])
def test_rows_that_begin_anywhere(gpu_lib, pm, dim, dtype):
    """Rows one after the other that begin on every element of a 16-byte word; what lies around them stays."""
    for n in (1, 2, 11, 300, 2500 if dim < 1000 else 1300):
        size = n * dim
        w, b = params(dim, torch.float32)
        for a in (0, 1, 3, 6, 7):
            x, grad = (rows((size + 16,), dtype, m, 1.0)[a:a + size].view(n, dim) for m in (0.2, 0.0))
            stats = torch.empty(n, 2, device="cuda")
            for c in (a, 2):   # (the output begins like the input, or does not)
                bufs = [torch.full((size + 16,), 7.0, device="cuda", dtype=dtype) for _ in range(2)]
                out, dx = (t[c:c + size].view(n, dim) for t in bufs)
                pm.layer_norm(x, w, b, out=out, stats=stats)
                into = gpu_lib.NormGrads(dx, torch.empty_like(w), torch.empty_like(b))
                pm.layer_norm_grad(x, grad, stats, w, out=into)
                pm.wait()
                check_forward(x, w, b, 1e-5, out, stats)
                check_grad(x, grad, stats, w, into)
                for t in bufs:
                    assert (t[:c] == 7).all() and (t[c + size:] == 7).all()
            y, g = x.clone().view(-1), grad
            flat = torch.full((size + 16,), 7.0, device="cuda", dtype=dtype)
            flat[a:a + size] = y
            over = flat[a:a + size].view(n, dim)
            pm.layer_norm(over, w, b, out=over)
            pm.wait()
            check_forward(x, w, b, 1e-5, over)
            assert (flat[:a] == 7).all() and (flat[a + size:] == 7).all()


@pytest.mark.parametrize("dim", [20, 256, 1003, 4096, 9001])
def test_in_place(gpu_lib, pm, dim):
    for dtype in DTYPES:
        x, grad = rows((77, dim), dtype), rows((77, dim), dtype)
        w, b = params(dim, torch.float32)
        stats = torch.empty(77, 2, device="cuda")
        out = pm.layer_norm(x, w, b, stats=stats)
        want = pm.layer_norm_grad(x, grad, stats, w)
        y, over_x, over_g = x.clone(), x.clone(), grad.clone()
        pm.layer_norm(y, w, b, out=y)
        dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
        a = pm.layer_norm_grad(over_x, grad, stats, w, out=gpu_lib.NormGrads(over_x, dw, None))
        b2 = pm.layer_norm_grad(x, over_g, stats, w, out=gpu_lib.NormGrads(over_g, None, db))
        pm.wait()
        assert torch.equal(y, out) and torch.equal(over_x, want.x) and torch.equal(over_g, want.x)
        assert torch.equal(dw, want.weight) and torch.equal(db, want.bias) and a.bias is None and b2.weight is None


def test_parts_of_the_gradient(gpu_lib, pm):
    x, grad = rows((50, 96), torch.float32), rows((50, 96), torch.float32)
    stats = torch.empty(50, 2, device="cuda")
    out = pm.layer_norm(x, stats=stats)
    pm.wait()
    check_forward(x, None, None, 1e-5, out, stats)
    got = pm.layer_norm_grad(x, grad, stats)
    assert got.weight is None and got.bias is None
    only_bias = pm.layer_norm_grad(x, grad, stats, bias=True, out=None)
    w, _ = params(96, torch.float32)
    no_bias = pm.layer_norm_grad(x, grad, stats, w, bias=False)
    nothing_else = pm.layer_norm_grad(x, grad, stats, w, out=gpu_lib.NormGrads(None, torch.empty(96, device="cuda"), None))
    pm.wait()
    check_grad(x, grad, stats, None, got)
    check_grad(x, grad, stats, None, only_bias)
    check_grad(x, grad, stats, w, no_bias)
    assert no_bias.bias is None and torch.equal(nothing_else.weight, no_bias.weight)


def test_no_rows(gpu_lib, pm):
    x = torch.empty(0, 40, device="cuda")
    w, b = params(40, torch.bfloat16)
    stats = torch.empty(0, 2, device="cuda")
    assert pm.layer_norm(x, w, b, stats=stats).shape == (0, 40)
    got = pm.layer_norm_grad(x, x, stats, w)
    pm.wait()
    assert got.x.shape == (0, 40) and not got.weight.any() and not got.bias.any()


@pytest.mark.parametrize("dim", [64, 1000, 5000, 30_000])
def test_large_means_and_constant_rows(gpu_lib, pm, dim):
    """A mean of 1000 deviations, rows of one value, and one element that is far from the others."""
    x = rows((40, dim), torch.float32, 1000.0, 1.0)
    x[7] = 3.25
    x[8] = 0.0
    x[9, 0] = -1e6
    stats = torch.empty(40, 2, device="cuda")
    out = pm.layer_norm(x, eps=1e-3, stats=stats)
    pm.wait()
    check_forward(x, None, None, 1e-3, out, stats)
    assert (out[8] == 0).all()


def test_what_is_no_number_stays_in_its_row(gpu_lib, pm):
    for dim in (48, 97, 1001, 3000, 10_000):
        x, stats = rows((20, dim), torch.bfloat16), torch.empty(20, 2, device="cuda")
        clean = pm.layer_norm(x, stats=stats)
        grad = rows((20, dim), torch.bfloat16)
        clean_dx = pm.layer_norm_grad(x, grad, stats).x
        x[3, 5], x[11, dim - 1], x[12, 0] = math.nan, math.inf, -math.inf
        grad[7, 0], grad[15, dim - 1] = math.nan, math.inf
        out = pm.layer_norm(x, stats=stats)
        dx = pm.layer_norm_grad(x, grad, stats).x
        pm.wait()
        bad = torch.zeros(20, dtype=torch.bool, device="cuda")
        bad[[3, 11, 12]] = True
        assert out[bad].isnan().all() and torch.equal(out[~bad], clean[~bad])
        bad[[7, 15]] = True
        assert (~torch.isfinite(dx[bad])).all() and torch.equal(dx[~bad], clean_dx[~bad])


def test_gradient_against_differences(gpu_lib, pm):
    """Central differences of sum(out * c) in 64 bits of the call's own outputs are too coarse; of the formula they are
    not: the gradient for out's gradient c against them."""
    torch.manual_seed(1)
    x, c = rows((3, 17), torch.float32), torch.randn(3, 17, device="cuda")
    w, b = params(17, torch.float32)
    stats = torch.empty(3, 2, device="cuda")
    pm.layer_norm(x, w, b, stats=stats)
    got = pm.layer_norm_grad(x, c, stats, w)
    pm.wait()
    f = lambda x, w, b: (forward64(x, w, b, 1e-5)[3] * c.double()).sum()   # noqa: E731
    step = 1e-5
    for t, g, at in ((x, got.x, (1, 4)), (x, got.x, (2, 16)), (w, got.weight, (3,)), (b, got.bias, (16,))):
        up, down = (t.double().clone() for _ in range(2))
        up[at] += step
        down[at] -= step
        args = lambda v: [v if q is t else q for q in (x, w, b)]   # noqa: E731
        slope = float(f(*args(up)) - f(*args(down))) / (2 * step)
        # (the differences err by step^2 of third derivatives, about 1e-8; the gradient as above)
        assert abs(float(g[at]) - slope) <= 1e-5 * max(1.0, abs(slope))


def test_recorded_in_a_graph_and_beside_another(gpu_lib):
    """Two graphs of one manager, launched in turn on new inputs, and eager calls between them."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        pm = gpu_lib.ParameterManager(4, 4, 1)
        w, b = params(300, torch.float32)
        sets = []
        for n in (50, 400):
            x, grad = rows((n, 300), torch.float16), rows((n, 300), torch.float16)
            out, stats = torch.empty_like(x), torch.empty(n, 2, device="cuda")
            into = gpu_lib.NormGrads(torch.empty_like(x), torch.empty_like(w), torch.empty_like(b))

            def call(x=x, grad=grad, out=out, stats=stats, into=into):
                pm.layer_norm(x, w, b, out=out, stats=stats)
                pm.layer_norm_grad(x, grad, stats, w, out=into)

            call()
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                call()
            sets.append((g, call, x, grad, out, stats, into))
        for _ in range(3):
            for g, call, x, grad, out, stats, into in sets:
                x.copy_(torch.randn(x.shape, device="cuda"))
                grad.copy_(torch.randn(x.shape, device="cuda"))
                g.replay()
                got = [t.clone() for t in (out, stats, *into)]
                call()
                torch.cuda.synchronize()
                for a, c in zip(got, (out, stats, *into)):
                    assert torch.equal(a, c)
        pm.close()


def test_the_same_bits_every_time(gpu_lib, pm):
    x, grad = rows((3000, 520), torch.bfloat16), rows((3000, 520), torch.bfloat16)
    w, b = params(520, torch.float32)
    stats = torch.empty(3000, 2, device="cuda")
    pm.layer_norm(x, w, b, stats=stats)
    first = pm.layer_norm_grad(x, grad, stats, w)
    for _ in range(5):
        again = pm.layer_norm_grad(x, grad, stats, w)
        pm.wait()
        assert all(torch.equal(a, c) for a, c in zip(first, again))


def test_refusals(gpu_lib, pm):
    x = torch.zeros(4, 8, device="cuda")
    stats = torch.zeros(4, 2, device="cuda")
    flat = torch.zeros(100, device="cuda")
    bad = [
        lambda: pm.layer_norm(x.cpu()),
        lambda: pm.layer_norm(x.double()),
        lambda: pm.layer_norm(x, torch.ones(7, device="cuda")),
        lambda: pm.layer_norm(x, torch.ones(8)),
        lambda: pm.layer_norm(x, eps=-1.0),
        lambda: pm.layer_norm(x, eps=math.nan),
        lambda: pm.layer_norm(x, out=torch.zeros(4, 9, device="cuda")),
        lambda: pm.layer_norm(x, out=torch.zeros(8, 4, device="cuda").t()),
        lambda: pm.layer_norm(x, out=flat.as_strided((4, 8), (4, 1))),           # overlapping rows
        lambda: pm.layer_norm(flat.as_strided((4, 8), (9, 1)), out=flat.as_strided((4, 8), (8, 1))),   # laid out anew
        lambda: pm.layer_norm(x, out=x.view(torch.float16)[:, :8]),
        lambda: pm.layer_norm(x, stats=torch.zeros(4, 1, device="cuda")),
        lambda: pm.layer_norm(x, stats=stats.half()),
        lambda: pm.layer_norm(torch.zeros(4, 0, device="cuda")),
        lambda: pm.layer_norm(torch.zeros((), device="cuda")),
        lambda: pm.layer_norm_grad(x, x[:3], stats),
        lambda: pm.layer_norm_grad(x, x, stats[:3]),
        lambda: pm.layer_norm_grad(x, x, stats.cpu()),
        lambda: pm.layer_norm_grad(x, x, stats, out=gpu_lib.NormGrads(torch.zeros(4, 9, device="cuda")[:, :7], None, None)),
        lambda: pm.layer_norm(x, flat[:8], out=flat.as_strided((4, 8), (8, 1))),   # over what the rows are scaled by
        lambda: pm.layer_norm(torch.zeros(4, 2, device="cuda"), out=stats, stats=stats),
        lambda: pm.layer_norm_grad(x, x.clone(), stats, flat[:8], out=gpu_lib.NormGrads(None, flat[:8], None)),
        lambda: pm.layer_norm_grad(x, x.clone(), stats, out=gpu_lib.NormGrads(None, flat[:8], flat[:8])),
        lambda: pm.layer_norm_grad(x, x.clone(), stats, out=gpu_lib.NormGrads(None, None, x[0])),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, gpu_lib.AdaPMError)) as e:
            call()
        assert not isinstance(e.value, gpu_lib.AdaPMError) or e.value.status == gpu_lib.EINVAL, i
    pm.wait()
    assert not flat.any() and not x.any()
    # what the call refuses leaves the manager as it was
    assert np.isfinite(pm.layer_norm(x).cpu().numpy()).all()


def test_offsets_beyond_32_bits(gpu_lib, pm):
    """More than 2^31 elements: the rows behind that are like the others."""
    n, dim = 530_000, 4096
    x = torch.empty(n, dim, dtype=torch.bfloat16, device="cuda")
    for a in range(0, n, 53_000):
        x[a:a + 53_000].normal_(0.5, 1.5)
    w, b = params(dim, torch.float32)
    stats = torch.empty(n, 2, device="cuda")
    out = pm.layer_norm(x, w, b, stats=stats)
    part = [0, 524_287, 524_288, 524_289, n - 1]
    pm.wait()
    check_forward(x[part], w, b, 1e-5, out[part], stats[part])
    got = pm.layer_norm_grad(x, out, stats, w)
    pm.wait()
    check_grad(x[part], out[part], stats[part], w, gpu_lib.NormGrads(got.x[part], None, None))
    want = out[:, 7].double() * (x[:, 7].double() - stats[:, 0].double()) * stats[:, 1].double()
    assert abs(float(got.weight[7].double() - want.sum())) <= (n / 152 + 300) * U * float(want.abs().sum())


def test_two_managers_at_once(gpu_lib):
    """Calls on two streams, side by side, with inputs that have to be copied first."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    pms = []
    for s in streams:
        with torch.cuda.stream(s):
            pms.append(gpu_lib.ParameterManager(4, 4, 1))
    w, b = params(700, torch.float32)
    xs = [torch.randn(700, 900, device="cuda").t() for _ in range(2)]        # (elements of a row lie apart)
    heavy = [torch.randn(3000, 4096, device="cuda").half() for _ in range(2)]
    weight = torch.randn(4096, 3000, device="cuda").half()
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        got = [(pm.layer_norm(x, w, b), pm.linear(h, weight, dtype=torch.float32)) for pm, x, h in zip(pms, xs, heavy)]
    for pm in pms:
        pm.wait()
    for (out, product), x, h in zip(got, xs, heavy):
        check_forward(x, w, b, 1e-5, out)
        want = h.double() @ weight.double()
        size = h.double().abs() @ weight.double().abs()
        assert ((product.double() - want).abs() <= (4096 / 8 + 16) * 2.0 ** -23 * size).all()
    for pm in pms:
        pm.close()
