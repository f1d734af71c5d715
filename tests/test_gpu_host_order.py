"""Pinned host arrays that one call fills and a later one reads, with no wait of the host in between: what is read is
what was written, in the order of the calls.  Each chain runs behind some 20 ms of other work on the library's stream,
so that a read in front of the write would find the array's old contents (valid keys and rows).  Values are dyadic:
sums are exact."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

K, D = 200, 16


def make(gpu_lib, **kw):
    init = (np.random.default_rng(3).integers(-64, 65, size=(K, D)) * 2.0 ** -5).astype(np.float32)
    return init, gpu_lib.ParameterManager(K, D, 1, init_values=torch.from_numpy(init).cuda(), **kw)


@pytest.fixture(scope="module")
def load():
    x = torch.zeros(1 << 28, device="cuda")

    def go():
        for _ in range(60):
            x.add_(1.0)
    return go


def pinned(a):
    return torch.as_tensor(a).pin_memory()


@pytest.mark.parametrize("into", [False, True])
@pytest.mark.parametrize("n", [60, 9000])
def test_gradient_rows_on_the_host_go_into_the_update(gpu_lib, load, n, into):
    init, pm = make(gpu_lib)
    rng = np.random.default_rng(n)
    t = rng.integers(0, K // 2, size=n)
    x = rng.integers(-8, 9, size=(n, D)) * 2.0 ** -3
    tokens, grad = pinned(t), pinned(x.astype(np.float32))
    out = gpu_lib.RowGrads(pinned(np.arange(n, dtype=np.int32) % K), pinned(np.full((n, D), 5.0, np.float32)),
                           pinned(np.zeros(1, np.int32))) if into else None
    torch.cuda.synchronize()
    load()
    g = pm.embed_grad(0, tokens, grad, scale=0.5, out=out)
    pm.push_grads(0, g.keys, g.rows, 0.25)
    pm.wait()
    want = init.astype(np.float64)
    np.add.at(want, t, -0.125 * x)
    assert np.array_equal(pm.read_main(np.arange(K)), want)
    pm.close()


@pytest.mark.parametrize("part", [slice(None), slice(30, 50), slice(63, 64)])
def test_pulled_rows_are_pushed(gpu_lib, load, part):
    """The whole of what a pull fills, and parts of it."""
    init, pm = make(gpu_lib)
    keys = np.random.default_rng(0).permutation(K)[:64]
    pk, rows = pinned(keys.astype(np.int32)), pinned(np.full((64, D), 7.0, np.float32))
    torch.cuda.synchronize()
    load()
    pm.pull(0, pk, out=rows)
    pm.push(0, pk[part], rows[part])
    pm.wait()
    want = init.copy()
    want[keys[part]] *= 2
    assert np.array_equal(pm.read_main(np.arange(K)), want)
    pm.close()


def test_looked_up_rows_are_a_gradient(gpu_lib, load):
    init, pm = make(gpu_lib)
    t = np.random.default_rng(1).integers(0, K, size=(5, 30))
    tokens, x = pinned(t), pinned(np.full((5, 30, D), 3.0, np.float32))
    torch.cuda.synchronize()
    load()
    pm.embed(0, tokens, scale=2.0, out=x)
    g = pm.embed_grad(0, tokens, x)
    pm.wait()
    keys, counts = np.unique(t, return_counts=True)
    assert np.array_equal(g.rows[:int(g.count)].numpy(), 2.0 * init[keys] * counts[:, None])
    pm.close()


def test_what_a_graph_fills_is_read_behind_it(gpu_lib, load):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        init, pm = make(gpu_lib)
        pk, rows = pinned(np.arange(0, K, 2, dtype=np.int32)), pinned(np.zeros((K // 2, D), np.float32))
        pm.pull(0, pk, out=rows)                                   # (the first call is in front of the capture)
        pm.wait()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            pm.pull(0, pk, out=rows)
        want = init.copy()
        for launch in range(3):
            pm.wait()
            rows.fill_(9.0)
            torch.cuda.synchronize()
            load()
            g.replay()
            pm.push(0, pk, rows)
            want[::2] *= 2
        pm.wait()
        assert np.array_equal(pm.read_main(np.arange(K)), want)
        pm.close()


def test_many_buffers_in_turn(gpu_lib):
    """More outputs than the library keeps track of at once, each read back by the next call."""
    init, pm = make(gpu_lib)
    keys = pinned(np.arange(K, dtype=np.int32))
    bufs = [pinned(np.zeros((K, D), np.float32)) for _ in range(200)]
    want = init.astype(np.float64)
    for i, b in enumerate(bufs + bufs):
        pm.pull(0, keys[:2], out=b[:2])
        pm.push(0, keys[2:4], b[:2])
        want[2:4] += want[:2]
    pm.wait()
    assert np.array_equal(pm.read_main(np.arange(K)), want)
    pm.close()
