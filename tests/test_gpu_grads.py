"""The gradient norm over many tensors, and clipping, against 64 bits.

Tolerances (u = 2^-24): at most 64 squares are added in fp32, each addition one rounding of a sum of positive terms
(64 u), the rest is fp64; the root halves that, and the result is rounded: 33 u of the norm.  A clipped element takes
the factor's two roundings and one product, 3 u, then one rounding to its type."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {torch.float32: (2.0 ** -24, 2.0 ** -149), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}


@pytest.fixture(scope="module")
def pm(gpu_lib):
    pm = gpu_lib.ParameterManager(4, 4, 1)
    yield pm
    pm.close()


def norm64(tensors, scale=1.0):
    return abs(scale) * math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))


def check(gpu_lib, pm, tensors, scale=1.0, limits=(0.3, 2.0)):
    """Norm, clipping out of place and in place."""
    want = norm64(tensors, scale)
    norm = pm.grad_norm(tensors, scale=scale)
    pm.wait()
    got = float(norm)
    assert abs(got - want) <= 33 * U * want
    for part in limits:
        limit = float(np.float32(part * want))
        outs = [torch.full_like(t, 7.0) for t in tensors]
        kept = [t.clone() for t in tensors]
        pm.clip_grads(tensors, norm, limit, scale=scale, out=outs)
        pm.wait()
        s = float(np.float32(scale))
        f = s * (1.0 if got <= limit else limit / got)
        for t, k, o in zip(tensors, kept, outs):
            assert torch.equal(t, k)
            y, (ut, tiny) = t.double() * f, TYPES[t.dtype]
            assert ((o.double() - y).abs() <= y.abs() * (3 * U * (1 + ut) + ut) + tiny).all()
        pm.clip_grads(tensors, norm, limit, scale=scale)      # in place: the same bits
        pm.wait()
        for t, o in zip(tensors, outs):
            assert torch.equal(t, o)
        for t, k in zip(tensors, kept):
            t.copy_(k)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 1023, 2048, 2049, 100_003, 3_000_000])
def test_one_tensor(gpu_lib, pm, dtype, n):
    check(gpu_lib, pm, [torch.randn(n, device="cuda").to(dtype)], scale=0.5)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_every_alignment_and_neighbours_stay(gpu_lib, pm, dtype):
    buf = torch.randn(20_000, device="cuda").to(dtype)
    for start in range(0, 9):
        for n in (1, 3, 5, 8, 13, 2047, 2050, 9001):
            t = buf[start:start + n]
            dst = torch.full((n + 24,), 3.0, device="cuda", dtype=dtype)
            keep = buf.clone()
            want = norm64([t])
            norm = pm.grad_norm([t])
            for shift in (start, (start + 1) % 8):
                dst.fill_(3.0)
                pm.clip_grads([t], norm, want / 2, out=[dst[8 + shift:8 + shift + n]])
                pm.wait()
                y = t.double() / 2
                ut, tiny = TYPES[dtype]
                assert ((dst[8 + shift:8 + shift + n].double() - y).abs() <= y.abs() * (ut + 40 * U) + tiny).all()
                assert (dst[:8 + shift] == 3.0).all() and (dst[8 + shift + n:] == 3.0).all()
            assert abs(float(norm) - want) <= 33 * U * want
            pm.clip_grads([t], norm, want / 2)
            pm.wait()
            assert torch.equal(buf[:start], keep[:start]) and torch.equal(buf[start + n:], keep[start + n:])
            buf.copy_(keep)


@pytest.mark.parametrize("count", [2, 31, 32, 33, 399, 400, 401, 900])
def test_many_tensors_of_every_type(gpu_lib, pm, count):
    rng = np.random.default_rng(count)
    tensors = []
    for i in range(count):
        dtype = list(TYPES)[i % 3]
        n = int(rng.integers(0, 40) if i % 5 else rng.integers(1000, 60_000))
        tensors.append(torch.randn(n + 9, device="cuda").to(dtype)[i % 9:i % 9 + n])
    check(gpu_lib, pm, tensors, scale=-0.25)


def test_nothing(gpu_lib, pm):
    for tensors in ([], [torch.empty(0, device="cuda")], [torch.zeros(5000, device="cuda")]):
        norm = pm.grad_norm(tensors)
        pm.clip_grads(tensors, norm, 0.0)
        pm.wait()
        assert float(norm) == 0.0 and not any(t.any() for t in tensors)


def test_outs_of_another_type(gpu_lib, pm):
    src = [torch.randn(5001, device="cuda").to(torch.bfloat16), torch.randn(77, device="cuda").to(torch.float16),
           torch.randn(4096, device="cuda")]
    outs = [torch.empty(5001, device="cuda"), torch.empty(77, device="cuda"),
            torch.empty(4096, device="cuda", dtype=torch.float16)]
    norm = pm.grad_norm(src, scale=1 / 8)
    pm.clip_grads(src, norm, 1.0, scale=1 / 8, out=outs)
    pm.wait()
    f = 1 / 8 / float(norm)
    for s, o in zip(src, outs):
        y, (ut, tiny) = s.double() * f, TYPES[o.dtype]
        assert ((o.double() - y).abs() <= y.abs() * (4 * U + ut) + tiny).all()


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e-3, 1e15, 1e25, 1e37])
def test_squares_beyond_fp32(gpu_lib, pm, size):
    """Norms whose squares overflow or vanish in fp32."""
    for n in (1, 64, 5000):
        t = torch.randn(n, device="cuda").abs().add(0.5) * size
        for u in (t, t.to(torch.bfloat16)):
            want = norm64([u])
            norm = pm.grad_norm([u])
            pm.wait()
            if want < 3e38:
                assert abs(float(norm) - want) <= 33 * U * want
            else:
                assert math.isinf(float(norm))
    mixed = [torch.full((300,), size, device="cuda"), torch.full((300,), 1.0, device="cuda")]
    want = norm64(mixed)
    norm = pm.grad_norm(mixed)
    pm.wait()
    assert abs(float(norm) - want) <= 33 * U * want


def test_small_beside_large_within_one_run(gpu_lib, pm):
    t = torch.full((4096,), 1e-30, device="cuda")
    t[17] = 1e20
    norm = pm.grad_norm([t])
    pm.wait()
    assert abs(float(norm) - 1e20) <= 33 * U * 1e20


@pytest.mark.parametrize("dtype", list(TYPES))
def test_infinities_and_nan_show(gpu_lib, pm, dtype):
    for bad in (float("inf"), -float("inf"), float("nan")):
        t = [torch.ones(3000, device="cuda", dtype=dtype), torch.ones(10, device="cuda", dtype=dtype)]
        t[0][2999] = bad
        norm = pm.grad_norm(t)
        outs = [torch.empty_like(x) for x in t]
        pm.clip_grads(t, norm, 1.0, out=outs)
        pm.wait()
        if math.isnan(bad):
            assert math.isnan(float(norm)) and all(bool(o.isnan().all()) for o in outs)
        else:
            assert math.isinf(float(norm)) and not outs[0][:2999].any() and bool(outs[0][2999].isnan())
    t = [torch.ones(10, device="cuda", dtype=dtype)]
    norm = pm.grad_norm(t)
    pm.clip_grads(t, norm, float("inf"))
    pm.wait()
    assert (t[0] == 1).all()


def test_rows_whose_number_the_device_knows(gpu_lib, pm):
    rows = torch.randn(50, 30, device="cuda")
    for live in (0, 1, 7, 50, 60):
        g = gpu_lib.RowGrads(torch.zeros(50, dtype=torch.int32, device="cuda"), rows.clone(),
                             torch.tensor([live], dtype=torch.int32, device="cuda"))
        g.rows[live:] = float("nan")                      # never looked at
        other = torch.randn(100, device="cuda")
        want = norm64([rows[:live], other])
        norm = pm.grad_norm([other, g])
        pm.clip_grads([other, g], norm, want / 4)
        pm.wait()
        assert abs(float(norm) - want) <= 33 * U * want
        assert torch.allclose(g.rows[:live], rows[:live] / 4, rtol=1e-5, atol=0)
        assert bool(g.rows[live:].isnan().all())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_whose_number_the_device_knows_into_others(gpu_lib, pm, dtype):
    rows, count = torch.randn(40, 21, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    keys = torch.zeros(40, dtype=torch.int32, device="cuda")
    for live in (0, 1, 13, 40, 41):
        count.fill_(live)
        src, dst = rows.clone(), torch.full((40, 21), 5.0, device="cuda", dtype=dtype)
        src[live:] = float("nan")
        more, out = torch.randn(77, device="cuda").to(dtype), torch.empty(77, device="cuda")
        want = norm64([rows[:live], more])
        g = gpu_lib.RowGrads(keys, src, count)
        norm = pm.grad_norm([g, more])
        # (the rows' number is the gradient's: the target's own is not looked at)
        for target in (dst, gpu_lib.RowGrads(keys, dst, torch.full_like(count, 3))):
            dst.fill_(5.0)
            pm.clip_grads([g, more], norm, want / 4, out=[target, out])
            pm.wait()
            ut, tiny = TYPES[dtype]
            y = rows[:live].double() / 4
            assert ((dst[:live].double() - y).abs() <= y.abs() * (ut + 40 * U) + tiny).all()
            assert (dst[live:] == 5.0).all()
            assert ((out.double() - more.double() / 4).abs() <= more.double().abs() * 40 * U).all()
        assert abs(float(norm) - want) <= 33 * U * want
        assert torch.equal(src[:live], rows[:live]) and bool(src[live:].isnan().all())


def test_the_same_every_time(gpu_lib, pm):
    t = [torch.randn(1_000_003, device="cuda"), torch.randn(500_000, device="cuda").to(torch.bfloat16)]
    norms = [pm.grad_norm(t) for _ in range(5)]
    pm.wait()
    assert len({float(n) for n in norms}) == 1


def test_more_than_2_to_the_32_elements(gpu_lib, pm):
    n = (1 << 32) + 12_345
    t = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    t[5], t[(1 << 31) + 7], t[n - 1] = 3.0, 4.0, 12.0
    norm = pm.grad_norm([t])
    pm.clip_grads([t], norm, 6.5)
    pm.wait()
    assert float(norm) == 13.0
    assert [float(t[5]), float(t[(1 << 31) + 7]), float(t[n - 1])] == [1.5, 2.0, 6.0]
    assert int((t != 0).sum()) == 3


def test_norms_that_are_no_aligned_float_are_refused(gpu_lib, pm):
    x, buf = torch.ones(10, device="cuda"), torch.zeros(8, device="cuda", dtype=torch.bfloat16)
    row, key = torch.zeros(1, 4, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for out in (buf[0], buf[1], x.double()[0], x[:2]):
        with pytest.raises(ValueError):
            pm.grad_norm([x], out=out)
    import ctypes
    lib = gpu_lib.load()
    t = gpu_lib._Tensor(x.data_ptr(), 10, None, 0, 0)
    for off in (1, 2, 3):
        at = buf.data_ptr() + off
        assert lib.adapm_grad_norm(pm._h, ctypes.byref(t), 1, 1.0, at) == gpu_lib.EINVAL
        assert lib.adapm_clip_grads(pm._h, ctypes.byref(t), None, 1, 1.0, 1.0, at) == gpu_lib.EINVAL
        assert lib.adapm_push_grads(pm._h, 0, key.data_ptr(), row.data_ptr(), 1, 4, 0, 0.1, 0.0, 1.0, 1.0,
                                    at) == gpu_lib.EINVAL
    host, scalar = torch.zeros(()).pin_memory(), torch.zeros(3, device="cuda")
    pm.grad_norm([x], out=host)
    pm.grad_norm([x], out=scalar[1])
    pm.wait()
    assert not buf.any() and scalar.tolist() == [0.0, float(host), 0.0] and abs(float(host) - math.sqrt(10)) < 1e-6
    assert (x == 1).all()


def test_refusals(gpu_lib, pm):
    x = torch.ones(10, device="cuda")
    norm = pm.grad_norm([x])
    for call in (lambda: pm.grad_norm([x.double()]), lambda: pm.grad_norm([x.cpu()]), lambda: pm.grad_norm([x[::2]]),
                 lambda: pm.clip_grads([x], norm, 1.0, out=[x, x]), lambda: pm.clip_grads([x], norm.cpu(), 1.0),
                 lambda: pm.clip_grads([x], norm.double(), 1.0)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: pm.clip_grads([x], norm, -1.0), lambda: pm.clip_grads([x], norm, float("nan")),
                 lambda: pm.clip_grads([x], norm, 1.0, out=[x[:5]]),
                 lambda: pm.clip_grads([x], norm, 1.0, out=[x.view(torch.bfloat16)[:10]])):
        with pytest.raises(gpu_lib.AdaPMError) as e:
            call()
        assert e.value.status == gpu_lib.EINVAL
    import ctypes
    lib = gpu_lib.load()
    host = np.ones(4, np.float32)
    for t in (gpu_lib._Tensor(x.data_ptr(), 10, None, 0, 5), gpu_lib._Tensor(None, 10, None, 0, 0),
              gpu_lib._Tensor(x.data_ptr() + 2, 5, None, 0, 0), gpu_lib._Tensor(host.ctypes.data, 4, None, 0, 0),
              gpu_lib._Tensor(x.data_ptr(), 1 << 50, None, 0, 0),
              gpu_lib._Tensor(x.data_ptr(), 10, host.ctypes.data, 1, 0)):
        assert lib.adapm_grad_norm(pm._h, ctypes.byref(t), 1, 1.0, norm.data_ptr()) == gpu_lib.EINVAL
    assert lib.adapm_grad_norm(pm._h, None, 1, 1.0, norm.data_ptr()) == gpu_lib.EINVAL
    assert lib.adapm_grad_norm(pm._h, None, 0, 1.0, None) == gpu_lib.EINVAL
    assert lib.adapm_grad_norm(None, None, 0, 1.0, norm.data_ptr()) == gpu_lib.EINVAL
    pm.wait()
    assert (x == 1).all()
