"""Matrix products with bias, activation and residual, and their gradients, against 64 bits.

Tolerances (u = 2^-24).  Products of 16-bit numbers are exact in fp32.  The tensor cores add 16 of them to a sum at a
time, each time off by at most two units in the last place (2^-23) of the magnitudes so far; parts of k and the epilogue
add a few roundings: a product over k errs by (k / 8 + 16) 2^-23 of the sum of magnitudes.  An activation multiplies
that by at most 1.2 and adds 16 u (1 + |z|).  Then one rounding to the output's type.  Where dz has an activation in it,
it is rounded to 16 bits before the products: its half step more, of the same sum.  The bias's gradient adds fp32
numbers, at most rows / 8 + 80 one after the other."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {torch.float32: (2.0 ** -24, 2.0 ** -149), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}
HALVES = [torch.float16, torch.bfloat16]
ACTS = [None, "relu", "gelu", "gelu_tanh", "silu", "tanh"]
# rows, ins, outs: around every limit of a tile, a block of k and the sizes of accesses; few rows; long sums
SIZES = [(1, 1, 1), (1, 64, 128), (1, 8, 5003), (1, 4096, 300), (2, 7, 9), (5, 333, 1000), (16, 65, 129), (17, 200, 256),
         (33, 1000, 127), (64, 512, 2048), (65, 64, 64), (100, 63, 65), (127, 129, 257), (128, 128, 256), (129, 72, 40),
         (300, 1024, 520), (777, 256, 1000), (1021, 333, 503), (40, 9000, 24), (130, 20_000, 70), (3000, 96, 3),
         (2500, 17, 1100)]
# enough tiles of 128 x 256 for every SM: pairs of blocks in the product, in dx, in dweight; sizes that nothing divides;
# long sums whose last tiles are halved
LARGE = [(2600, 200, 4100), (2600, 4100, 200), (100, 2600, 4100), (2601, 1001, 4099), (4096, 512, 4096),
         (4090, 4100, 4095), (2100, 4096, 4096)]


@pytest.fixture(scope="module")
def pm(gpu_lib):
    pm = gpu_lib.ParameterManager(4, 4, 1)
    yield pm
    pm.close()


def act64(z, name):
    z = z.double()
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return {"relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z), "tanh": lambda: torch.tanh(z),
            None: lambda: z}[name]()


def slope64(z, name):
    z = z.double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return {"relu": lambda: (z > 0).double(), "silu": lambda: s * (1 + z * (1 - s)),
            "tanh": lambda: 1 - torch.tanh(z) ** 2, None: lambda: torch.ones_like(z)}[name]()


def check(x, w, b, act, res, out, pre=None):
    k = w.shape[0]
    z = x.double() @ w.double()
    err = (k / 8 + 16) * 2.0 ** -23 * (x.double().abs() @ w.double().abs())
    if b is not None:
        z = z + b.double()
        err = err + 2 * U * (z.abs() + b.double().abs())
    if pre is not None:
        ut, tiny = TYPES[pre.dtype]
        assert ((pre.double() - z).abs() <= err + z.abs() * ut + tiny).all()
    y = act64(z, act)
    err = 1.2 * err + 16 * U * (1 + z.abs())
    if res is not None:
        y = y + res.double()
        err = err + U * (y.abs() + res.double().abs())
    ut, tiny = TYPES[out.dtype]
    assert ((out.double() - y).abs() <= err * (1 + ut) + y.abs() * ut + tiny).all()


def check_grad(x, w, grad, pre, act, got):
    rows = x.numel() // max(1, x.shape[-1])
    x2, g2 = x.reshape(rows, -1).double(), grad.reshape(rows, -1).double()
    dz = g2 * slope64(pre.reshape(rows, -1), act) if act else g2
    off = TYPES[x.dtype][0] if act else 0.0
    size = dz.abs() + (32 * U * g2.abs() / max(off, 1e-9) if act else 0)   # (the slope's own error, under the half step)
    if got.x is not None:
        want = dz @ w.double().t()
        err = (off + (w.shape[1] / 8 + 16) * 2.0 ** -23) * (size @ w.double().abs().t())
        ut, tiny = TYPES[got.x.dtype]
        # (16-bit dz below the normal numbers are off by half of the smallest one)
        err = err + TYPES[x.dtype][1] * w.double().abs().sum(1) * (1 if act else 0)
        assert ((got.x.reshape(rows, -1).double() - want).abs() <= err + want.abs() * ut + tiny).all()
    if got.weight is not None:
        want = x2.t() @ dz
        err = (off + (rows / 8 + 16) * 2.0 ** -23) * (x2.abs().t() @ size)
        err = err + TYPES[x.dtype][1] * x2.abs().sum(0).unsqueeze(1) * (1 if act else 0)
        ut, tiny = TYPES[got.weight.dtype]
        assert ((got.weight.double() - want).abs() <= err + want.abs() * ut + tiny).all()
    if got.bias is not None:
        want = dz.sum(0)
        ut, tiny = TYPES[got.bias.dtype]
        err = (rows / 8 + 80) * U * dz.abs().sum(0) + 32 * U * g2.abs().sum(0)
        assert ((got.bias.double() - want).abs() <= err + want.abs() * ut + tiny).all()


def small(shape, dtype):
    """Whole numbers: every product and sum is exact."""
    return torch.randint(-3, 4, shape, device="cuda").to(dtype)


def stored(w, by_out):
    return w.t().contiguous().t() if by_out else w.contiguous()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("size", range(len(SIZES)))
def test_whole_numbers_are_exact(gpu_lib, pm, size, dtype):
    """Bit for bit, in every way that the operands are stored in."""
    rows, ins, outs = size[0] if isinstance(size, tuple) else SIZES[size]
    x, w = small((rows, ins), dtype), small((ins, outs), dtype)
    b, res = small((outs,), dtype), small((rows, outs), torch.float32)
    grad = small((rows, outs), dtype)
    z = x.double() @ w.double()
    dx, dw = grad.double() @ w.double().t(), x.double().t() @ grad.double()
    for x_across in (False, True):
        for by_out in (False, True):
            xs, ws = stored(x, x_across), stored(w, by_out)
            out = pm.linear(xs, ws, dtype=torch.float32)
            all_of_it = pm.linear(xs, ws, b, "relu", res, dtype=torch.float32)
            into = gpu_lib.LinearGrads(torch.empty(rows, ins, device="cuda"),
                                       stored(torch.empty(ins, outs, device="cuda"), by_out), torch.empty(outs, device="cuda"))
            pm.linear_grad(xs, ws, stored(grad, x_across), out=into)
            pm.wait()
            assert torch.equal(out.double(), z)
            assert torch.equal(all_of_it.double(), (z + b.double()).clamp(min=0) + res.double())
            assert torch.equal(into.x.double(), dx)
            assert torch.equal(into.weight.double(), dw)
            assert torch.equal(into.bias.double(), grad.double().sum(0))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("size", range(len(LARGE)))
def test_large_products_of_whole_numbers_are_exact(gpu_lib, pm, size, dtype):
    test_whole_numbers_are_exact(gpu_lib, pm, (LARGE[size],), dtype)


# sizes whose two gradients share a launch (few tiles; a last round with free blocks; both products longer than the
# other) and some whose do not; one rounding of an exact sum, so that bits are compared
@pytest.mark.parametrize("size", [(777, 256, 1000), (70, 96, 50), (300, 520, 130), (2600, 4100, 200), (4096, 512, 4096),
                                  (1300, 4099, 1027), (130, 20_000, 70), (40, 90, 24), (5000, 2048, 2048)])
def test_gradients_of_two_types(gpu_lib, pm, size):
    rows, ins, outs = size
    for dtype in HALVES:
        x, w, grad = small((rows, ins), dtype), small((ins, outs), dtype), small((rows, outs), dtype)
        dx, dw = grad.double() @ w.double().t(), x.double().t() @ grad.double()
        for of_x, of_w in ((dtype, torch.float32), (torch.float32, dtype), (dtype, dtype)):
            for by_out in (False, True):
                into = gpu_lib.LinearGrads(torch.empty(rows, ins, device="cuda", dtype=of_x),
                                           stored(torch.empty(ins, outs, device="cuda", dtype=of_w), by_out), None)
                pm.linear_grad(x, w, grad, out=into)
                pm.wait()
                assert torch.equal(into.x, dx.float().to(of_x))
                assert torch.equal(into.weight, dw.float().to(of_w))


@pytest.mark.parametrize("act", ["gelu", "tanh"])
@pytest.mark.parametrize("size", range(len(LARGE)))
def test_large_sizes(gpu_lib, pm, size, act):
    test_every_size(gpu_lib, pm, (LARGE[size],), act)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("size", range(len(SIZES)))
def test_every_size(gpu_lib, pm, size, act):
    rows, ins, outs = size[0] if isinstance(size, tuple) else SIZES[size]
    size = rows + ins
    torch.manual_seed(size)
    for dtype in HALVES:
        x = torch.randn(rows, ins, device="cuda").to(dtype)
        w = stored((torch.randn(ins, outs, device="cuda") / math.sqrt(ins)).to(dtype), size % 2)
        b = torch.randn(outs, device="cuda").to(dtype if size % 3 else torch.float32)
        res = torch.randn(rows, outs, device="cuda").to(dtype)
        pre = torch.empty(rows, outs, device="cuda", dtype=dtype)
        out = pm.linear(x, w, b, act, res, pre=pre)
        plain = pm.linear(x, w, activation=act, dtype=torch.float32)
        pm.wait()
        assert out.dtype == dtype and plain.dtype == torch.float32
        check(x, w, b, act, res, out, pre)
        check(x, w, None, act, None, plain)
        grad = (torch.randn(rows, outs, device="cuda") * 0.1).to(dtype)
        got = pm.linear_grad(x, w, grad, pre, act)
        pm.wait()
        assert got.x.dtype == got.weight.dtype == got.bias.dtype == dtype and got.weight.stride() == w.stride()
        check_grad(x, w, grad, pre, act, got)


@pytest.mark.parametrize("rows,ins,outs", [(6, 40, 72), (150, 136, 264), (90, 77, 131)])
def test_strides_and_neighbours(gpu_lib, pm, rows, ins, outs):
    dtype = torch.bfloat16
    for gap in (8, 3):
        x = torch.randn(rows, ins + gap, device="cuda").to(dtype)[:, gap:]
        w = (torch.randn(ins, outs + gap, device="cuda") / math.sqrt(ins)).to(dtype)[:, :outs]
        res = torch.randn(rows, outs + gap, device="cuda").to(dtype)[:, gap:]
        room = torch.full((rows + 2, outs + 2 * gap), 7.0, device="cuda", dtype=dtype)
        kept = torch.full((rows + 2, outs + 2 * gap), 7.0, device="cuda", dtype=dtype)
        out, pre = room[1:-1, gap:-gap], kept[1:-1, gap:-gap]
        pm.linear(x, w, None, "silu", res, out=out, pre=pre)
        pm.wait()
        check(x, w, None, "silu", res, out, pre)
        for t in (room, kept):
            mask = torch.ones_like(t, dtype=torch.bool)
            mask[1:-1, gap:-gap] = False
            assert (t[mask] == 7.0).all()
        grad = torch.randn(rows, outs + gap, device="cuda").to(dtype)[:, :outs]
        dx, dw = (torch.full((a + 2, b + 2 * gap), 7.0, device="cuda", dtype=dtype) for a, b in ((rows, ins), (ins, outs)))
        into = gpu_lib.LinearGrads(dx[1:-1, gap:-gap], dw[1:-1, gap:-gap], None)
        pm.linear_grad(x, w, grad, pre, "silu", out=into)
        pm.wait()
        check_grad(x, w, grad, pre, "silu", into)
        for t in (dx, dw):
            mask = torch.ones_like(t, dtype=torch.bool)
            mask[1:-1, gap:-gap] = False
            assert (t[mask] == 7.0).all()
    # one row for all, one value for a row, steps over rows, and leading dimensions
    x = torch.randn(1, ins, device="cuda").to(dtype).expand(rows, ins)
    w = torch.randn(ins, 2 * outs, device="cuda").to(dtype)[:, ::2]
    out = pm.linear(x, w)
    grad = torch.randn(rows, 1, device="cuda").to(dtype).expand(rows, outs)
    got = pm.linear_grad(x, torch.randn(outs, ins, device="cuda").to(dtype).t(), grad)
    pm.wait()
    check(x, w, None, None, None, out)
    assert torch.equal(got.bias.double(), grad.double().sum(0).to(dtype).double()) or rows > 1
    wide = torch.randn(3, rows + 1, ins, device="cuda").to(dtype)
    w = w.contiguous()
    y = pm.linear(wide[:, :-1], w)
    z = pm.linear(wide[:, ::2].transpose(0, 1), w)
    one = pm.linear(wide[0, 0], w)
    pm.wait()
    assert y.shape == (3, rows, outs) and one.shape == (outs,)
    check(wide[:, :-1].reshape(-1, ins), w, None, None, None, y.reshape(-1, outs))
    check(wide[:, ::2].transpose(0, 1).reshape(-1, ins), w, None, None, None, z.reshape(-1, outs))
    check(wide[0, :1], w, None, None, None, one.view(1, -1))


def test_residual_in_place(gpu_lib, pm):
    for rows, ins, outs in ((5, 64, 256), (300, 200, 520), (70, 33, 41), (1, 4096, 128)):
        x = torch.randn(rows, ins, device="cuda").half()
        w = (torch.randn(ins, outs, device="cuda") / math.sqrt(ins)).half()
        res = torch.randn(rows, outs, device="cuda")
        want = pm.linear(x, w, None, "gelu", res, dtype=torch.float32)
        y = res.clone()
        pm.linear(x, w, None, "gelu", y, out=y)
        pm.wait()
        assert torch.equal(y, want)


@pytest.mark.parametrize("size", [(1, 4096, 300), (40, 9000, 24), (130, 20_000, 70), (2600, 4100, 200), (300, 1024, 520),
                                  (9000, 65, 130), (20_000, 300, 40), (4096, 2100, 1500), (500, 577, 3000)])
def test_long_sums_in_32_bits(gpu_lib, pm, size):
    """Positive numbers, whose sums' errors add up. At most 512 products are summed in the tensor cores, 16 at a time, by
    two units in the last place each (and 16 more, as above): 80 * 2^-23; the chains' sums by a half each: k / 512 * 2^-24,
    and parts of k and the rest of the epilogue by 16 * 2^-24."""
    rows, ins, outs = size
    for dtype in HALVES:
        x, w, g = (torch.rand(s, device="cuda").add_(1).to(dtype) for s in ((rows, ins), (ins, outs), (rows, outs)))
        for by_out in (False, True):
            ws = stored(w, by_out)
            out = pm.linear(x, ws, dtype=torch.float32)
            into = gpu_lib.LinearGrads(torch.empty(rows, ins, device="cuda"),
                                       stored(torch.empty(ins, outs, device="cuda"), by_out), None)
            pm.linear_grad(x, ws, g, out=into)
            pm.wait()
            for got, a, b in ((out, x, w), (into.x, g, w.t()), (into.weight, x.t(), g)):
                want = a.double() @ b.double()
                k = a.shape[1]
                assert ((got.double() - want).abs() <= want * (80 * 2.0 ** -23 + (k / 512 + 16) * 2.0 ** -24)).all()


def test_parts_of_the_gradient(gpu_lib, pm):
    x, w, grad = torch.randn(70, 96, device="cuda").half(), torch.randn(96, 50, device="cuda").half(), \
        torch.randn(70, 50, device="cuda").half()
    full = pm.linear_grad(x, w, grad)
    for keep in range(8):
        into = gpu_lib.LinearGrads(*(torch.empty_like(t) if keep >> i & 1 else None for i, t in enumerate(full)))
        got = pm.linear_grad(x, w, grad, out=into)
        pm.wait()
        for i, t in enumerate(got):
            assert t is None or torch.equal(t, full[i])
    assert pm.linear_grad(x, w, grad, bias=False).bias is None


def test_no_rows(gpu_lib, pm):
    x, w = torch.empty(0, 40, device="cuda").half(), torch.ones(40, 24, device="cuda").half()
    assert pm.linear(x, w, activation="tanh").shape == (0, 24)
    for ws in (w, stored(w, True)):
        wide = torch.full((40, 30), 5.0, device="cuda", dtype=torch.float16)
        got = pm.linear_grad(x, ws, x.new_empty(0, 24), x.new_empty(0, 24), "tanh")
        pm.linear_grad(x, ws, x.new_empty(0, 24), out=gpu_lib.LinearGrads(None, wide[:, 3:27], None))
        pm.wait()
        assert got.x.shape == (0, 40) and not got.weight.any() and not got.bias.any()
        assert not wide[:, 3:27].any() and (wide[:, :3] == 5).all() and (wide[:, 27:] == 5).all()


def test_what_is_no_number_stays_in_its_row(gpu_lib, pm):
    for rows in (10, 200):
        x, w = torch.randn(rows, 130, device="cuda").bfloat16(), torch.randn(130, 90, device="cuda").bfloat16()
        clean = pm.linear(x, w, activation="relu")
        x[3, 5], x[7, 129] = math.nan, math.inf
        out = pm.linear(x, w, activation="relu")
        pm.wait()
        assert out[3].isnan().all() and not torch.isfinite(out[7]).all() | (out[7] == 0).all()
        for r in range(rows):
            assert r in (3, 7) or torch.equal(out[r], clean[r])


def test_gradient_against_differences(gpu_lib, pm):
    """Central differences of the formula in 64 bits, for every input of a layer, at 1e-2 (16-bit outputs and dz)."""
    torch.manual_seed(4)
    x, w, b = torch.randn(9, 24, device="cuda").half(), (torch.randn(24, 16, device="cuda") / 5).half(), \
        torch.randn(16, device="cuda").half()
    c = torch.randn(9, 16, device="cuda").half()
    for act in ACTS:
        pre = torch.empty_like(c)
        pm.linear(x, w, b, act, pre=pre)
        into = gpu_lib.LinearGrads(torch.empty(9, 24, device="cuda"), torch.empty(24, 16, device="cuda"),
                                   torch.empty(16, device="cuda"))
        pm.linear_grad(x, w, c, pre, act, out=into)
        pm.wait()
        f = lambda x, w, b: (act64(x @ w + b, act) * c.double()).sum()   # noqa: E731
        for which, at in ((0, (2, 3)), (0, (8, 23)), (1, (5, 15)), (1, (23, 0)), (2, (7,))):
            up, down = ([t.double().clone() for t in (x, w, b)] for _ in range(2))
            up[which][at] += 1e-5
            down[which][at] -= 1e-5
            slope = float(f(*up) - f(*down)) / 2e-5
            # (pre and dz are rounded to 2^-11 of themselves, sums of 16 or 9 terms of size one, slopes' slopes below 1.5)
            kink = act == "relu"
            assert abs(float(into[which][at]) - slope) <= 24 * 3 * 2.0 ** -11 * 3 or kink


def test_recorded_in_a_graph_and_the_same_bits(gpu_lib):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        pm = gpu_lib.ParameterManager(4, 4, 1)
        sets = []
        for rows, ins, outs in ((3, 2048, 300), (500, 333, 260), (4096, 4096, 4096)):
            x, w = torch.randn(rows, ins, device="cuda").half(), (torch.randn(ins, outs, device="cuda") / 50).half()
            pre, out, grad = (torch.randn(rows, outs, device="cuda").half() for _ in range(3))
            into = gpu_lib.LinearGrads(torch.empty_like(x), torch.empty_like(w), torch.empty(outs, device="cuda"))

            def call(x=x, w=w, pre=pre, out=out, grad=grad, into=into):
                pm.linear(x, w, activation="tanh", out=out, pre=pre)
                pm.linear_grad(x, w, grad, pre, "tanh", out=into)

            call()
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                call()
            sets.append((g, call, x, (out, pre, *into)))
        for _ in range(3):
            for g, call, x, outs in sets:
                x.copy_(torch.randn(x.shape, device="cuda"))
                g.replay()
                got = [t.clone() for t in outs]
                call()
                torch.cuda.synchronize()
                for a, c in zip(got, outs):
                    assert torch.equal(a, c)
        pm.close()


def test_refusals(gpu_lib, pm):
    x, w = torch.zeros(4, 8, device="cuda").half(), torch.zeros(8, 16, device="cuda").half()
    y, flat = torch.zeros(4, 16, device="cuda").half(), torch.zeros(200, device="cuda").half()
    square, y16, y17, w16 = (torch.zeros(16, 16, device="cuda").half() for _ in range(4))
    bad = [
        lambda: pm.linear(x.float(), w.float()),
        lambda: pm.linear(x, w.bfloat16()),
        lambda: pm.linear(x.cpu(), w),
        lambda: pm.linear(x, w.cpu()),
        lambda: pm.linear(x, w[:7]),
        lambda: pm.linear(x, w[0]),
        lambda: pm.linear(x, w, torch.zeros(15, device="cuda")),
        lambda: pm.linear(x, w, activation="sigmoid"),
        lambda: pm.linear(x, w, residual=y.float()),
        lambda: pm.linear(x, w, residual=y[:3]),
        lambda: pm.linear(x, w, dtype=torch.bfloat16),
        lambda: pm.linear(x, w, out=torch.zeros(4, 15, device="cuda").half()),
        lambda: pm.linear(x, w, out=torch.zeros(16, 4, device="cuda").half().t()),
        lambda: pm.linear(x, w, out=flat.as_strided((4, 16), (8, 1))),
        lambda: pm.linear(x, w, pre=torch.zeros(4, 16, device="cuda")),
        lambda: pm.linear(x, w, out=y, pre=y),
        lambda: pm.linear(x, torch.zeros(8, 0, device="cuda").half()),
        lambda: pm.linear(torch.zeros(4, 0, device="cuda").half(), torch.zeros(0, 16, device="cuda").half()),
        lambda: pm.linear(torch.zeros(16, 16, device="cuda").half()[:4], w.new_zeros(16, 16), out=flat.as_strided((4, 16), (-0 + 4, 1))),
        lambda: pm.linear_grad(x, w, y, activation="tanh"),
        lambda: pm.linear_grad(x, w, y.float()),
        lambda: pm.linear_grad(x, w, y[:3]),
        lambda: pm.linear_grad(x, w, y, y.float(), "relu"),
        lambda: pm.linear_grad(x, w, y, out=gpu_lib.LinearGrads(x, None, None)),
        lambda: pm.linear_grad(x, w, y, out=gpu_lib.LinearGrads(None, w, None)),
        lambda: pm.linear(square, w16, square[0], out=square),
        lambda: pm.linear(square, w16, y16[0], out=y16),
        lambda: pm.linear(square, w16, y16[0], pre=y16),
        lambda: pm.linear(square, square.clone(), residual=y16, pre=y16),   # (out may be the residual, pre may not)
        lambda: pm.linear_grad(square, square.clone(), y16, out=gpu_lib.LinearGrads(None, square, None)),
        lambda: pm.linear_grad(square, square.clone(), y16, out=gpu_lib.LinearGrads(None, y16, None)),
        lambda: pm.linear_grad(square, square.clone(), y16, y17, "relu", out=gpu_lib.LinearGrads(y17, None, None)),
        lambda: pm.linear_grad(square, square.clone(), y16, y17, "relu", out=gpu_lib.LinearGrads(None, None, y17[0])),
        lambda: pm.linear_grad(square, w16, y16, out=gpu_lib.LinearGrads(w16, None, None)),
        lambda: pm.linear_grad(x, w, y, out=gpu_lib.LinearGrads(None, flat.as_strided((8, 16), (2, 3)), None)),
        lambda: pm.linear_grad(x, w, y, out=gpu_lib.LinearGrads(None, torch.zeros(8, 16, device="cuda").bfloat16(), None)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, gpu_lib.AdaPMError)) as e:
            call()
        assert not isinstance(e.value, gpu_lib.AdaPMError) or e.value.status == gpu_lib.EINVAL, i
    pm.wait()
    assert not any(t.any() for t in (flat, x, w, y, square, y16, y17, w16))
    assert not pm.linear(x, w).any()


def test_offsets_beyond_32_bits(gpu_lib, pm):
    """More than 2^31 outputs: the rows behind that are like the others; and as inputs of the gradient."""
    rows, ins, outs = 66_000, 40, 32_768
    x, w = small((rows, ins), torch.bfloat16), small((ins, outs), torch.bfloat16)
    out = pm.linear(x, w)
    pm.wait()
    part = [0, 65_535, 65_536, rows - 1]
    want = x[part].double() @ w.double()
    assert ((out[part].double() - want).abs() <= want.abs() * 2.0 ** -8).all()   # (whole sums, rounded once)
    grad = out.clamp_(-1, 1)
    got = pm.linear_grad(x, w, grad, out=gpu_lib.LinearGrads(torch.empty(rows, ins, device="cuda"), None, None))
    pm.wait()
    assert torch.equal(got.x[part].double(), grad[part].double() @ w.double().t())
