"""Token embeddings through the C ABI against plain implementations in 64 bits: lookup with scaling, its gradient by
sorted tokens, and the update by gradient rows.

Tolerances (u = 2^-24, half the spacing of fp32 at 1):
  * a looked-up row is one product of the pulled row, rounded once: bit-equal to the same product formed elsewhere;
  * a sum of m fp32 terms in any order errs by at most (m - 1) u times the sum of magnitudes to first order, the scale
    by u of the result: (m + 1) u sum |x| |scale|, with a factor 1.01 for the higher orders.  Sums of dyadic rows are
    exact;
  * an update's factor takes two roundings, its product with the row one, the learning rate one: 4 u of the step;
    with AdaGrad g*g has 7 u, the radicand 2 more, its inverse root half of these and u, the products 3 u: below
    16 u; the value's own rounding is u of the larger of the old and the new value, taken as 2 u of their sum.
"""
import numpy as np
import pytest
import torch

from oracle import ParameterManagerOracle

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def table(K, D, seed=0):
    return np.random.default_rng(seed).normal(0, 0.1, size=(K, D)).astype(np.float32)


def make(gpu_lib, init, W=1, **kw):
    return gpu_lib.ParameterManager(init.shape[0], init.shape[1], W, init_values=torch.from_numpy(init).cuda(), **kw)


def zipf(n, K, seed=0, s=1.2):
    """Tokens with a few hot ones."""
    rng = np.random.default_rng(seed)
    return np.minimum(rng.pareto(s, size=n) * 3, 2.0 ** 40).astype(np.int64) * 7919 % K


# -- lookup ---------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,dim", [(4, 1), (4, 4), (8, 7), (36, 36), (52, 50), (64, 64), (200, 100), (300, 299),
                                   (512, 512), (1024, 1023), (1024, 1024)])
@pytest.mark.parametrize("n", [1, 2, 31, 1000])
def test_lookup_is_the_scaled_rounded_row(gpu_lib, dtype, D, dim, n):
    K = 97
    init = table(K, D)
    pm = make(gpu_lib, init)
    t = torch.from_numpy(zipf(n, K, n)).cuda()
    want = (torch.from_numpy(init)[t.cpu()][:, :dim] * np.float32(1.7)).to(dtype)
    for ids in (t, t.to(torch.int32)):
        got = pm.embed(0, ids, dim, scale=1.7, dtype=dtype)
        pm.wait()
        assert got.shape == (n, dim) and got.dtype == dtype
        assert torch.equal(got.cpu(), want)
    pm.close()


# either end of every width that the kernel has lanes and loads for, rows of a multiple of eight elements or not
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [8, 32, 40, 64, 72, 128, 136, 256, 264, 512, 520, 640, 768, 776, 1024,
                                 2, 14, 18, 31, 33, 62, 66, 127, 129, 254, 258, 381, 386, 449, 510, 514, 767, 770, 1021])
def test_lookup_of_every_width(gpu_lib, dtype, dim):
    K, D = 97, -(-dim // 8) * 8
    init = table(K, D)
    pm = make(gpu_lib, init)
    for n in (3, 70, 30_000):   # (a warp's batch: one round of rows, some, as many as it takes)
        t = zipf(n, K, n)
        want = (torch.from_numpy(init[:, :dim]) * np.float32(-0.3)).to(dtype)[torch.from_numpy(t)]
        buf = torch.full((n * dim + 8,), 9.0, device="cuda", dtype=dtype)
        for first in (0, 1, 2, 4):   # rows that begin on every vector boundary and between them
            buf.fill_(9.0)
            pm.embed(0, torch.from_numpy(t).cuda(), dim, scale=-0.3, out=buf[first:first + n * dim].view(n, dim))
            pm.wait()
            assert torch.equal(buf[first:first + n * dim].view(n, dim).cpu(), want)
            assert (buf[:first] == 9.0).all() and (buf[first + n * dim:] == 9.0).all()
    pm.close()


def test_lookup_of_strided_tokens_into_strided_rows(gpu_lib):
    K, D, dim = 1000, 64, 60
    init = table(K, D)
    pm = make(gpu_lib, init)
    full = torch.from_numpy(zipf(7 * 41, K).reshape(7, 41)).cuda()
    wide = torch.full((7, 50, 80), -5.0, device="cuda", dtype=torch.bfloat16)
    cases = [
        (full[:, :-1], wide[:, 3:43, :dim]),                       # inner and outer gaps, aligned and not
        (full[:, 1:], wide[:, :40, 17:17 + dim]),
        (full[::2, ::3], wide[:4, :28:2, :dim]),
        (full.t(), wide[:, :41, :dim].transpose(0, 1)),            # rows in another order
        (full[:, 5], wide[:, 0, :dim]),
        (full[3:4, :4], wide[3:4, :4, :dim]),
        (full[:, :40].view(7, 8, 5), wide[:, :40, :dim].unflatten(1, (8, 5))),
        (full[0], None),
        (full[:, :1], wide[:, :1, 1:1 + dim]),
    ]
    for i, (t, out) in enumerate(cases):
        expect = wide.clone()
        got = pm.embed(0, t, dim, scale=-2.5, out=out, dtype=torch.bfloat16)
        pm.wait()
        want = (torch.from_numpy(init)[t.cpu()][..., :dim] * -2.5).to(torch.bfloat16)
        assert torch.equal(got.cpu(), want), f"case {i}"
        if out is not None:   # nothing else was written
            expect.as_strided(out.shape, out.stride(), out.storage_offset()).copy_(want)
            assert torch.equal(wide, expect), f"case {i}: elsewhere"
    pm.close()


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("pad", [0, 5, -1, -100, 10 ** 6])
def test_padding_has_zero_rows_and_is_no_error(gpu_lib, ids, pad):
    K, D = 50, 12
    init = table(K, D)
    pm = make(gpu_lib, init)
    t = torch.from_numpy(zipf(200, K)).to(ids)
    t[::7] = pad
    got = pm.embed(0, t.cuda(), scale=3.0, pad=pad)
    pm.wait()                                                     # (no ADAPM_ERANGE)
    want = torch.from_numpy(init)[t.long().clamp(0, K - 1)] * 3.0
    want[t == pad] = 0.0
    assert torch.equal(got.cpu(), want)
    pm.close()


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("pad", [2 ** 32, 2 ** 32 + 3, -2 ** 32 + 3, -2 ** 31 - 1, 2 ** 40 + 7, -2 ** 63, 2 ** 63 - 1,
                                 2 ** 64, 2 ** 64 + 3, -2 ** 64 + 7])
def test_padding_that_no_id_can_equal_pads_nothing(gpu_lib, ids, pad):
    """A pad beyond the ids' type is none of them: not the token that its low bits spell."""
    K, D, n = 50, 12, 200
    init = table(K, D)
    pm = make(gpu_lib, init)
    t = torch.from_numpy(zipf(n, K)).to(ids)
    t[::5], t[1::5] = pad & 31, 0
    got = pm.embed(0, t.cuda(), scale=3.0, pad=pad)
    g = pm.embed_grad(0, t.cuda(), torch.ones(n, D, device="cuda"), pad=pad)
    pm.wait()
    assert torch.equal(got.cpu(), torch.from_numpy(init)[t.long()] * 3.0)
    keys, counts = np.unique(t.numpy(), return_counts=True)
    check_row_grads(g, keys, np.repeat(counts[:, None], D, 1).astype(np.float64), 0.0)
    pm.close()


@pytest.mark.parametrize("ids,bad", [(torch.int32, 50), (torch.int32, -1), (torch.int64, 50), (torch.int64, -1),
                                     (torch.int64, 2 ** 32), (torch.int64, 2 ** 32 + 3), (torch.int64, -2 ** 40)])
@pytest.mark.parametrize("n", [40, 20_000])
def test_ids_outside_the_store_are_reported_and_count_as_padding(gpu_lib, ids, bad, n):
    K, D = 50, 8
    init = table(K, D)
    pm = make(gpu_lib, init)
    t = torch.from_numpy(zipf(n, K)).to(ids)
    t[3] = bad
    got = pm.embed(0, t.cuda())
    with pytest.raises(gpu_lib.AdaPMError) as e:
        pm.wait()
    assert e.value.status == gpu_lib.ERANGE
    assert not got[3].any() and torch.equal(got[4:].cpu(), torch.from_numpy(init)[t[4:].long()])
    grad = torch.ones(n, D, device="cuda")
    g = pm.embed_grad(0, t.cuda(), grad)
    with pytest.raises(gpu_lib.AdaPMError) as e:
        pm.wait()
    assert e.value.status == gpu_lib.ERANGE
    t[3] = t[4]
    keys, counts = np.unique(np.delete(t.numpy(), 3), return_counts=True)
    check_row_grads(g, keys, np.repeat(counts[:, None], D, 1).astype(np.float64), 0.0)
    pm.close()


@pytest.mark.parametrize("relocate,refresh", [(False, False), (True, False), (False, True)])
def test_lookup_reads_what_pull_reads_in_every_replica_state(gpu_lib, relocate, refresh):
    K, D, W = 300, 20, 3
    init = table(K, D)
    pm = make(gpu_lib, init, W, relocate=relocate, delta_refresh=refresh)
    ref = ParameterManagerOracle(K, D, W, init)
    rng = np.random.default_rng(1)
    every = torch.arange(K, device="cuda")

    def same():
        for w in range(W):
            assert torch.equal(pm.embed(w, every, scale=0.5), pm.pull(w, every) * 0.5)
        pm.wait()

    same()
    for clock in range(4):
        for w in range(W):
            keys = rng.integers(0, K, size=80)
            pm.intent(w, torch.from_numpy(keys).cuda(), clock, clock + 2)
            same()
            for times in range(2):
                d = rng.normal(size=(60, D)).astype(np.float32)
                pm.push(w, torch.from_numpy(keys[:60]).cuda(), torch.from_numpy(d).cuda())
                same()
        if clock % 2:
            pm.sync()
            same()
        for w in range(W):
            pm.advance_clock(w)
            same()
    assert not np.array_equal(pm.read_main(np.arange(K)), ref.read_main(np.arange(K)))
    pm.close()


@pytest.mark.parametrize("D", [8, 64, 200, 256, 600, 1024])
@pytest.mark.parametrize("relocate,refresh", [(False, False), (True, False), (False, True)])
def test_wide_loads_read_what_pull_reads_in_every_replica_state(gpu_lib, D, relocate, refresh):
    """Rows of a multiple of eight floats: aliases, pending updates, replicas with values of their own, folded ones."""
    K, W = 90, 2
    pm = make(gpu_lib, table(K, D), W, relocate=relocate, delta_refresh=refresh)
    rng = np.random.default_rng(D)
    every = torch.arange(K, device="cuda")

    def same():
        for w in range(W):
            rows = pm.pull(w, every)
            for dtype in TYPES:
                got = pm.embed(w, every, scale=0.5, dtype=dtype)
                pm.wait()
                assert torch.equal(got, (rows * 0.5).to(dtype))

    same()
    for clock in range(3):
        for w in range(W):
            pm.intent(w, torch.from_numpy(rng.integers(0, K, size=50)).cuda(), clock, clock + 2)
            for times in range(3):
                keys = torch.from_numpy(rng.integers(0, K, size=40)).cuda()
                pm.push(w, keys, torch.from_numpy(rng.normal(size=(40, D)).astype(np.float32)).cuda())
                same()
        if clock == 1:
            pm.sync()
            same()
        for w in range(W):
            pm.advance_clock(w)
            same()
    assert not np.array_equal(pm.read_main(np.arange(K)), table(K, D))
    pm.close()


def test_lookup_with_early_events_and_on_the_host(gpu_lib):
    """A lookup is a worker's first access of a clock as a pull is; host ids and rows are taken as everywhere."""
    K, D = 200, 16
    init = table(K, D)
    pm = make(gpu_lib, init)
    t = torch.from_numpy(zipf(64, K))
    for clock in range(3):
        pm.intent(0, t.cuda(), clock + 1, clock + 2)
        pm.embed(0, t.cuda())
        pm.advance_clock(0)
    pm.wait()
    assert pm.stats()["early_advances"] >= 2
    want = torch.from_numpy(init)[t] * 2.0
    for ids in (t, t.to(torch.int32), t.pin_memory(), t.numpy(), t.reshape(8, 8)):
        got = pm.embed(0, ids, scale=2.0, dtype=torch.float16)
        pm.wait()
        assert not got.is_cuda and torch.equal(got.reshape(64, D), want.to(torch.float16))
    g = pm.embed_grad(0, t, torch.ones(64, D))
    pm.wait()
    keys, counts = np.unique(t.numpy(), return_counts=True)
    check_row_grads(g, keys, np.repeat(counts[:, None], D, 1).astype(np.float64), 0.0)
    assert not g.rows[len(keys):].any()
    pm.close()


def test_host_arrays_with_gaps_are_refused_whatever_else_is_on_the_host(gpu_lib):
    pm = make(gpu_lib, table(20, 8))
    t, x = torch.arange(12).reshape(3, 4), torch.ones(3, 4, 16)
    for call in (lambda: pm.embed(0, t[:, :3].clone(), out=x[:, :3, :8]), lambda: pm.embed(0, t[:, :3], out=torch.ones(3, 3, 8)),
                 lambda: pm.embed_grad(0, t, x[:, :, :8]), lambda: pm.embed_grad(0, t[:, :3], torch.ones(3, 3, 8))):
        with pytest.raises(gpu_lib.AdaPMError) as e:
            call()
        assert e.value.status == gpu_lib.EINVAL and "gaps" in str(e.value)
    pm.wait()
    pm.close()


# -- gradient -------------------------------------------------------------------
def check_row_grads(g, keys, sums, bound):
    """g holds `keys` and sums within `bound`, then no keys."""
    n = int(g.count.cpu())
    assert n == len(keys)
    got = g.keys.cpu().numpy()
    assert np.array_equal(got[:n].astype(np.int64) & 0xFFFFFFFF, keys)
    assert (got[n:] == -1).all()
    assert (np.abs(g.rows.cpu().numpy()[:n].astype(np.float64) - sums) <= bound).all()


def plain_grad(tokens, grad, scale, drop=()):
    """Distinct tokens, sums, sums of magnitudes and occurrences in 64 bits."""
    keep = ~np.isin(tokens, list(drop))
    keys, inv, m = np.unique(tokens[keep], return_inverse=True, return_counts=True)
    out = np.zeros((2, len(keys), grad.shape[1]))
    np.add.at(out[0], inv, grad[keep] * scale)
    np.add.at(out[1], inv, np.abs(grad[keep] * scale))
    return keys, out[0], out[1], m


def check_grad(gpu_lib, K, tokens, dim, dtype, ids=torch.int64, pad=None, scale=1.3, D=None, pm=None, dyadic=False,
               seed=0):
    """embed_grad of tokens (numpy) with random rows against 64 bits."""
    rng = np.random.default_rng(seed)
    n = tokens.size
    x = rng.integers(-64, 65, size=(n, dim)) * 2.0 ** -7 if dyadic else rng.normal(size=(n, dim))
    grad = torch.from_numpy(x).to(dtype)
    own = pm is None
    if own:
        pm = make(gpu_lib, np.zeros((K, D or -(-dim // 4) * 4), np.float32))
    scale = 0.5 if dyadic else scale
    g = pm.embed_grad(0, torch.from_numpy(tokens).to(ids).cuda(), grad.cuda(), scale=scale, pad=pad)
    pm.wait()
    keys, sums, mags, m = plain_grad(tokens.reshape(-1), grad.double().numpy(), float(np.float32(scale)),
                                     () if pad is None else (pad,))
    check_row_grads(g, keys, sums, 0.0 if dyadic else 1.01 * (m[:, None] + 1) * U * mags)
    if own:
        pm.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [1, 3, 4, 8, 12, 16, 25, 50, 64, 96, 100, 200, 256, 300, 333, 512, 600, 768, 1000, 1023,
                                 1024])
@pytest.mark.parametrize("n", [1, 5, 700])
def test_gradient_sums_the_rows_of_equal_tokens(gpu_lib, dtype, dim, n):
    check_grad(gpu_lib, 500, zipf(n, 500, dim), dim, dtype, dyadic=dim % 2 == 0)


# one block's span, several, the counting sort's end, several chunks and spans per key, a single key throughout
@pytest.mark.parametrize("n", [33, 64, 2047, 8191, 8192, 8193, 20_011, 100_000])
@pytest.mark.parametrize("K,s", [(1, 1.2), (2, 1.2), (300, 0.6), (100_000, 1.2), (100_000, 0.2)])
def test_gradient_of_every_length_and_skew(gpu_lib, n, K, s):
    check_grad(gpu_lib, K, zipf(n, K, n, s), 24, torch.bfloat16, ids=torch.int32 if n % 2 else torch.int64)
    check_grad(gpu_lib, K, zipf(n, K, n, s), 24, torch.float32, dyadic=True)


@pytest.mark.parametrize("n,dim", [(300_000, 64), (70_000, 512), (1_000_000, 16), (50_000, 333)])
def test_gradient_of_large_batches(gpu_lib, n, dim):
    check_grad(gpu_lib, 70_000, zipf(n, 70_000, n, 0.9), dim, torch.float16, dyadic=True)


def test_gradient_of_more_spans_than_a_block_sums(gpu_lib):
    check_grad(gpu_lib, 3_000_000, zipf(5_000_000, 3_000_000, 4, 0.7), 4, torch.float32, ids=torch.int32, dyadic=True)


# either side of where another sort takes over, and of where its tiles grow
@pytest.mark.parametrize("n", [6143, 6144, 6145, 65_536, 65_537, 131_071, 131_072, 131_073, 262_145,
                               524_288, 524_289])
@pytest.mark.parametrize("K", [3, 256, 257, 65_536, 1_000_000, 20_000_000])
def test_gradient_by_every_sort(gpu_lib, n, K):
    t = zipf(n, K, n, 0.4)
    t[::11] = -1
    check_grad(gpu_lib, K, t, 4, torch.bfloat16, ids=torch.int32 if n % 2 else torch.int64, pad=-1, dyadic=True)


@pytest.mark.parametrize("n", [100, 30_000])
@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("pad", [0, 17, -1, -100, 10 ** 6])
def test_gradient_leaves_padding_out(gpu_lib, n, ids, pad):
    t = zipf(n, 60, 3)
    t[::3] = pad
    check_grad(gpu_lib, 60, t, 20, torch.float32, ids=ids, pad=pad)


@pytest.mark.parametrize("n", [64, 9000])
def test_gradient_of_padding_alone_is_empty(gpu_lib, n):
    check_grad(gpu_lib, 60, np.full(n, 7), 20, torch.bfloat16, ids=torch.int32, pad=7)
    check_grad(gpu_lib, 60, np.full(n, -1), 20, torch.bfloat16, pad=-1)


def test_empty_batches(gpu_lib):
    pm = make(gpu_lib, table(10, 8))
    t = torch.empty((3, 0), dtype=torch.int64, device="cuda")
    assert pm.embed(0, t).shape == (3, 0, 8)
    g = pm.embed_grad(0, t, torch.empty((3, 0, 8), device="cuda"))
    pm.push_grads(0, g.keys, g.rows, 0.1)
    pm.wait()
    assert int(g.count) == 0 and g.keys.numel() == 0
    pm.close()


def test_gradient_of_strided_and_broadcast_rows(gpu_lib):
    K, dim = 90, 40
    pm = make(gpu_lib, np.zeros((K, dim), np.float32))
    full = torch.from_numpy(zipf(12 * 33, K).reshape(12, 33)).cuda()
    wide = torch.randn(12, 40, 56, device="cuda", dtype=torch.float32)
    cases = [
        (full[:, :-1], wide[:, 2:34, :dim]),
        (full[:, 1:], wide[:, :32, 5:5 + dim]),                            # unaligned rows
        (full.t(), wide[:, :33, :dim].transpose(0, 1)),
        (full, wide[:1, :33, :dim].expand(12, 33, dim)),                   # one row for all sequences
        (full, wide[:, :1, :dim].expand(12, 33, dim)),                     # one row for all positions
        (full, wide[0, 0, :dim].expand(12, 33, dim)),
        (full, wide[:, :33, :1].expand(12, 33, dim)),                      # one value for all elements
        (full[::3, ::2], wide[:4, :17, :dim].to(torch.bfloat16)),
        (full.view(12, 3, 11), wide[:, :33, :dim].unflatten(1, (3, 11))),
        (full.view(12, 3, 11).transpose(0, 2), wide[:, :33, :dim].unflatten(1, (3, 11)).transpose(0, 2)),
    ]
    for i, (t, grad) in enumerate(cases):
        g = pm.embed_grad(0, t, grad, scale=0.7)
        pm.wait()
        keys, sums, mags, m = plain_grad(t.reshape(-1).cpu().numpy(), grad.reshape(-1, dim).double().cpu().numpy(),
                                         float(np.float32(0.7)))
        check_row_grads(g, keys, sums, 1.01 * (m[:, None] + 1) * U * mags)
    pm.close()


def test_gradient_is_that_of_the_lookup(gpu_lib):
    """Differences of sum(weights * embed(tokens)) as single store elements move; dyadic values, exact in fp32."""
    K, D, n = 12, 8, 50
    rng = np.random.default_rng(5)
    init = (rng.integers(-32, 33, size=(K, D)) * 2.0 ** -5).astype(np.float32)
    weights = torch.from_numpy(rng.integers(-8, 9, size=(n, D)) * 2.0 ** -3).float().cuda()
    t = torch.from_numpy(zipf(n, K)).cuda()
    pm = make(gpu_lib, init)

    def loss():
        x = pm.embed(0, t, scale=4.0)
        pm.wait()
        return float((x.double() * weights.double()).sum())

    g = pm.embed_grad(0, t, weights, scale=4.0)
    pm.wait()
    dense = np.zeros((K, D))
    dense[g.keys[:int(g.count)].cpu().numpy()] = g.rows[:int(g.count)].cpu().numpy()
    base = loss()
    for k in range(K):
        for c in range(0, D, 3):
            step = torch.zeros(1, D, device="cuda")
            step[0, c] = 0.25
            pm.push(0, torch.tensor([k], device="cuda"), step)
            assert (loss() - base) / 0.25 == dense[k, c], (k, c)
            pm.push(0, torch.tensor([k], device="cuda"), -step)
    pm.close()


@pytest.mark.parametrize("n", [3000, 20_000])
@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
def test_gradient_takes_an_intents_plan(gpu_lib, n, ids):
    """Tokens that were signalled are grouped by the intent's plan, others by a sort; the same bits either way."""
    K, dim = 700, 32
    rng = np.random.default_rng(n)
    t = torch.from_numpy(zipf(n, K)).to(ids).cuda()
    other = torch.from_numpy(zipf(n, K, 9)).to(ids).cuda()
    grad = torch.from_numpy(rng.normal(size=(n, dim))).to(torch.bfloat16).cuda()
    plain, pm = (make(gpu_lib, np.zeros((K, dim), np.float32)) for _ in range(2))
    pm.intent(0, t, 0, 5)
    for tokens, misses in ((t, 0), (other, 1), (t, 1)):
        for pad in (None, int(t[0])):
            a = pm.embed_grad(0, tokens, grad, pad=pad)
            b = plain.embed_grad(0, tokens, grad, pad=pad)
            pm.wait()
            plain.wait()
            u = int(a.count)
            assert u == int(b.count) and torch.equal(a.keys, b.keys) and torch.equal(a.rows[:u], b.rows[:u])
    st = pm.stats()
    assert st["planned_pushes"] == 6 and st["plan_misses"] >= 2 and plain.stats()["planned_pushes"] == 0
    pm.close()
    plain.close()


@pytest.mark.parametrize("n", [3000, 20_000, 600_000])   # (by counting, by the token sort, by the push's sort)
@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("view", ["flat", "shifted", "transposed", "host"])
def test_a_signalled_batch_hits_its_plan_and_another_misses(gpu_lib, n, ids, view):
    """Each call's own count of plans looked up and missed, whatever layout and type the tokens have."""
    K, dim = 700, 4

    def batch(seed):
        t = torch.from_numpy(zipf(n // 8 * 8 + 8, K, seed)).to(ids).reshape(8, -1).cuda()
        return {"flat": t[:, :n // 8].contiguous(), "shifted": t[:, :-1], "transposed": t[:, 1:].t(),
                "host": t[:, :-1].contiguous().cpu()}[view]

    pm = make(gpu_lib, np.zeros((K, dim), np.float32))
    t, other = batch(1), batch(2)
    pm.intent(0, t, 0, 5)
    pm.wait()
    grad = torch.ones((*t.shape, dim), device="cuda")
    planned = missed = 0
    for tokens, hit in ((t, True), (other, False), (t, True)):
        for pad in (None, -1, K, int(t[0, 0]), int(other[0, 0])):   # (no token's, or a valid one's)
            g = pm.embed_grad(0, tokens, grad, pad=pad)
            pm.wait()
            st = pm.stats()
            planned, missed = planned + 1, missed + (not hit)
            assert st["planned_pushes"] == planned and st["plan_misses"] == missed
            keys, counts = np.unique(tokens.cpu().numpy(), return_counts=True)
            keep = keys != pad
            check_row_grads(g, keys[keep], np.repeat(counts[keep][:, None], dim, 1).astype(np.float64), 0.0)
    pm.close()


def test_gradient_is_the_same_every_time(gpu_lib):
    K, dim, n = 5000, 100, 60_000
    pm = make(gpu_lib, np.zeros((K, dim), np.float32))
    t = torch.from_numpy(zipf(n, K)).cuda()
    grad = torch.randn(n, dim, device="cuda")
    runs = [pm.embed_grad(0, t, grad) for _ in range(3)]
    pm.wait()
    u = int(runs[0].count)
    for r in runs[1:]:
        assert torch.equal(r.rows[:u], runs[0].rows[:u]) and torch.equal(r.keys, runs[0].keys)
    pm.close()


def test_infinities_and_nan_stay_with_their_token(gpu_lib):
    pm = make(gpu_lib, np.zeros((10, 8), np.float32))
    t = torch.tensor([3, 1, 3, 2, 9, 9, 5], device="cuda")
    grad = torch.ones(7, 8, device="cuda")
    grad[0, 2], grad[3, 5], grad[4, 1], grad[5, 1], grad[6] = float("inf"), float("nan"), float("inf"), -float("inf"), float("nan")
    g = pm.embed_grad(0, t, grad, pad=5)     # (padding's rows may hold anything)
    pm.wait()
    want = torch.ones(4, 8)
    want[2] = 2.0
    want[3] = 2.0
    want[2, 2], want[1, 5], want[3, 1] = float("inf"), float("nan"), float("nan")
    assert g.keys[:4].tolist() == [1, 2, 3, 9]
    assert torch.equal(torch.nan_to_num(g.rows[:4].cpu(), nan=-7.0), torch.nan_to_num(want, nan=-7.0))
    pm.close()


# -- update ---------------------------------------------------------------------
def plain_update(v, rows, dim, lr, factor, adagrad, eps):
    """New values, the step and its bound in 64 bits."""
    v, g = v.astype(np.float64), rows.astype(np.float64) * factor
    step = np.zeros_like(v)
    if adagrad:
        a = v[:, dim:]
        step[:, :dim] = -lr * g / np.sqrt(a + g * g + eps)
        step[:, dim:] = g * g
    else:
        step[:, :dim] = -lr * g
    return v + step, 2 * U * (np.abs(v) + np.abs(v + step)) + 16 * U * np.abs(step) + 1e-38


@pytest.mark.parametrize("adagrad", [False, True])
@pytest.mark.parametrize("dim", [4, 8, 20, 36, 64, 100, 128, 150, 200, 256, 300, 400, 512])
@pytest.mark.parametrize("state", ["main", "replica", "pushed twice", "others hold it", "relocated"])
def test_update_applies_rows_as_the_formula(gpu_lib, adagrad, dim, state):
    K, n, W = 400, 150, 3
    if adagrad and dim % 4:
        dim += 2
    D = 2 * dim if adagrad else -(-dim // 4) * 4
    rng = np.random.default_rng(dim)
    init = table(K, D, dim)
    if adagrad:
        init[:, dim:] = rng.uniform(0.01, 1.0, size=(K, dim))
    pm = make(gpu_lib, init, W, relocate=state == "relocated")
    keys = np.sort(rng.choice(K, size=n, replace=False))
    dk = torch.from_numpy(keys).to(torch.int32).cuda()
    every = torch.arange(K, device="cuda")
    if state in ("replica", "pushed twice", "relocated"):
        pm.intent(0, dk[::2], 0, 3)
    if state in ("others hold it", "relocated"):
        pm.intent(1, dk[::3], 0, 3)
        pm.intent(2, every, 0, 3)
    if state == "pushed twice":
        for _ in range(2):
            pm.push(0, dk[:n // 2], torch.full((n // 2, D), 0.01, device="cuda"))
    for times in range(3):
        before = pm.pull(0, every).cpu().numpy()
        others = [pm.pull(w, every).cpu().numpy() for w in (1, 2)]
        rows = rng.normal(size=(n, dim)).astype(np.float32)
        norm, max_norm = (None, 1.0) if times == 0 else (torch.tensor(3.7 if times == 1 else 0.2, device="cuda"), 1.0)
        pm.push_grads(0, dk, torch.from_numpy(rows).cuda(), 0.05, adagrad=adagrad, scale=0.25, norm=norm,
                      max_norm=max_norm)
        after = pm.pull(0, every).cpu().numpy()
        pm.wait()
        factor = 0.25 / (float(norm) if times == 1 else 1.0)
        want, bound = plain_update(before[keys], rows, dim, float(np.float32(0.05)), factor, adagrad,
                                   float(np.float32(1e-8)))
        assert (np.abs(after[keys] - want) <= bound).all()
        rest = np.setdiff1d(np.arange(K), keys)
        assert np.array_equal(after[rest], before[rest])
        if state == "others hold it":   # a write to main leaves other workers' replicas as they were until a sync
            for w, old in zip((1, 2), others):
                now = pm.pull(w, every).cpu().numpy()
                held = keys[::3] if w == 1 else np.arange(K)
                assert np.array_equal(now[held], old[held])
    pm.sync()
    final = pm.pull(0, every).cpu().numpy()
    assert np.allclose(final, after, rtol=1e-4, atol=1e-5)   # merged: the same sums, other roundings
    pm.close()


@pytest.mark.parametrize("D,dim", [(52, 50), (4, 1), (12, 9), (64, 33), (1024, 999)])
def test_update_of_the_first_floats_of_a_row(gpu_lib, D, dim):
    K, n = 100, 40
    init = table(K, D)
    pm = make(gpu_lib, init)
    keys = np.arange(1, 2 * n, 2)
    rows = np.random.default_rng(0).normal(size=(n, dim)).astype(np.float32)
    pm.push_grads(0, torch.from_numpy(keys).cuda(), torch.from_numpy(rows).cuda(), 0.5)
    pm.wait()
    want, bound = plain_update(init[keys], rows, dim, 0.5, 1.0, False, 0.0)
    got = pm.read_main(np.arange(K))
    assert (np.abs(got[keys] - want) <= bound).all() and np.array_equal(got[keys][:, dim:], init[keys][:, dim:])
    assert np.array_equal(np.delete(got, keys, 0), np.delete(init, keys, 0))
    pm.close()


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("bad", ["nan norm", "infinite norm", "nan scale", "infinite lr", "nan row"])
@pytest.mark.parametrize("D,dim", [(52, 50), (64, 32), (12, 9), (12, 1), (300, 100), (1024, 516), (1024, 999)])
def test_update_leaves_what_lies_behind_dim(gpu_lib, D, dim, bad, held):
    """Factors and rows that are no numbers reach the first dim floats only, zeros of either sign included."""
    K, n = 60, 25
    init = table(K, D)
    init[::2, dim:] = 0.0
    init[1::2, dim + 1:] = -0.0
    pm = make(gpu_lib, init)
    keys = np.arange(1, 2 * n, 2)
    dk = torch.from_numpy(keys).cuda()
    if held:
        pm.intent(0, dk, 0, 9)
    rows = torch.ones(n, dim, device="cuda")
    kw = dict(norm=torch.tensor({"nan norm": np.nan, "infinite norm": np.inf}.get(bad, 2.0), device="cuda"), max_norm=1.0)
    lr = np.inf if bad == "infinite lr" else 0.5
    if bad == "nan scale":
        kw["scale"] = float("nan")
    if bad == "nan row":
        rows[:, 0] = float("nan")
    for times in range(3):   # (a replica's first push, its second, and later ones are written differently)
        pm.push_grads(0, dk, rows, lr, **kw)
        got = pm.pull(0, torch.arange(K, device="cuda")).cpu().numpy()
        pm.wait()
        assert np.array_equal(got[:, dim:].view(np.uint32), init[:, dim:].view(np.uint32)), times
        if bad != "infinite norm":
            assert not np.isfinite(got[keys, 0]).any()
        else:
            assert np.array_equal(got[keys, :dim], init[keys, :dim])
    pm.sync()
    got = pm.read_main(np.arange(K))
    assert np.array_equal(got[:, dim:].view(np.uint32), init[:, dim:].view(np.uint32))
    pm.close()


@pytest.mark.parametrize("adagrad", [False, True])
def test_update_by_an_infinite_norm(gpu_lib, adagrad):
    """Nothing changes but where an infinity or a NaN came from."""
    K, dim = 30, 12
    init = np.abs(table(K, 2 * dim if adagrad else dim)) + 0.1
    pm = make(gpu_lib, init)
    rows = torch.ones(8, dim, device="cuda")
    rows[2, 5], rows[6, 0] = float("inf"), float("nan")
    pm.push_grads(0, torch.arange(3, 11, device="cuda"), rows, 0.5, adagrad=adagrad,
                  norm=torch.tensor(float("inf"), device="cuda"), max_norm=1.0)
    pm.wait()
    want = init.copy()
    for k, c in ((5, 5), (9, 0)):
        want[k, c] = float("nan")
        if adagrad:
            want[k, dim + c] = float("nan")
    assert np.array_equal(pm.read_main(np.arange(K)), want, equal_nan=True)
    pm.close()


def test_buffers_of_a_larger_batch(gpu_lib):
    """The last, smaller batch in the buffers of the others: nothing of theirs is updated again."""
    K, D = 50, 8
    init = table(K, D)
    pm = make(gpu_lib, init)
    ones = torch.ones(20, D, device="cuda")
    buf = pm.embed_grad(0, torch.arange(20, 40, device="cuda"), ones)
    g = pm.embed_grad(0, torch.tensor([3, 3, 1], device="cuda"), ones[:3], out=buf)
    assert g.keys.shape == (3,) and g.rows.shape == (3, D)
    norm = pm.grad_norm([g])
    pm.push_grads(0, g.keys, g.rows, 1.0)
    pm.wait()
    want = init.copy()
    want[1] -= 1
    want[3] -= 2
    assert np.array_equal(pm.read_main(np.arange(K)), want)
    assert abs(float(norm) - np.sqrt(5 * D)) < 1e-5
    pm.close()


@pytest.mark.parametrize("dim", [4, 64])
def test_rows_that_begin_between_vectors(gpu_lib, dim):
    """Gradient rows, and the rows of sums, whose first element is on no vector boundary."""
    K, n = 80, 300
    init = table(K, dim)
    pm = make(gpu_lib, init)
    t = zipf(n, K)
    x = torch.randn(n * dim + 1, device="cuda")[1:].view(n, dim)
    out = gpu_lib.RowGrads(torch.empty(n, dtype=torch.int32, device="cuda"),
                           torch.zeros(n * dim + 1, device="cuda")[1:].view(n, dim),
                           torch.empty(1, dtype=torch.int32, device="cuda"))
    pm.embed_grad(0, torch.from_numpy(t).cuda(), x, out=out)
    pm.push_grads(0, out.keys, out.rows, 0.5)
    pm.wait()
    keys, sums, mags, m = plain_grad(t, x.double().cpu().numpy(), 1.0)
    check_row_grads(out, keys, sums, 1.01 * (m[:, None] + 1) * U * mags)
    want, bound = plain_update(init[keys], out.rows[:len(keys)].cpu().numpy(), dim, 0.5, 1.0, False, 0.0)
    assert (np.abs(pm.read_main(keys) - want) <= bound).all()
    pm.close()


@pytest.mark.parametrize("refresh", [False, True])
def test_update_equals_a_push_of_the_formed_rows(gpu_lib, refresh):
    """The same bits as adapm_push of -lr * g, in every replica state, over several clocks."""
    K, D, W, n = 500, 24, 3, 120
    a, b = (make(gpu_lib, table(K, D), W, delta_refresh=refresh) for _ in range(2))
    rng = np.random.default_rng(2)
    for clock in range(6):
        for w in range(W):
            keys = torch.from_numpy(np.sort(rng.choice(K, size=n, replace=False))).to(torch.int32).cuda()
            rows = torch.from_numpy(rng.normal(size=(n, D)).astype(np.float32)).cuda()
            for pm in (a, b):
                pm.intent(w, keys[::2], clock + 1, clock + 3)
            a.push_grads(w, keys, rows, 0.125, scale=0.5)
            b.push(w, keys, rows * 0.5 * -0.125)
        for pm in (a, b):
            if clock % 2:
                pm.sync()
            for w in range(W):
                pm.advance_clock(w)
            pm.wait()
        k = np.arange(K)
        assert np.array_equal(a.read_main(k), b.read_main(k))
        for w in range(W):
            for x, y in zip(a.replica_rows(w, k), b.replica_rows(w, k)):
                assert np.array_equal(x, y)
    a.close()
    b.close()


def test_update_skips_missing_keys_and_reports_bad_ones(gpu_lib):
    K, D = 50, 8
    init = table(K, D)
    pm = make(gpu_lib, init)
    one = torch.ones(6, D, device="cuda")

    def go(keys):
        pm.push_grads(0, torch.tensor(keys, dtype=torch.int32, device="cuda"), one, 1.0)
        pm.wait()

    go([3, 7, 9, -1, -1, -1])
    got = pm.read_main(np.arange(K))
    want = init.copy()
    want[[3, 7, 9]] -= 1
    assert np.array_equal(got, want)
    for keys, status, touched in (([1, 2, 2, 4, 5, 6], gpu_lib.ESTATE, [1, 2, 4, 5, 6]),
                                  ([1, 2, 4, 3, 8, 9], gpu_lib.ESTATE, [1, 2, 4, 8, 9]),
                                  ([1, 2, 4, 5, 6, 50], gpu_lib.ERANGE, [1, 2, 4, 5, 6])):
        with pytest.raises(gpu_lib.AdaPMError) as e:
            go(keys)
        assert e.value.status == status
        want[touched] -= 1
        assert np.array_equal(pm.read_main(np.arange(K)), want)
    pm.close()


# -- the calls as calls ---------------------------------------------------------
def test_refusals(gpu_lib):
    pm = make(gpu_lib, table(20, 16), 2)
    t = torch.arange(6, device="cuda")
    x = torch.zeros(6, 16, device="cuda")

    def refused(kind, call, *words):
        with pytest.raises(kind) as e:
            call()
        if kind is gpu_lib.AdaPMError:
            assert e.value.status == gpu_lib.EINVAL
        for w in words:
            assert w in str(e.value), str(e.value)

    E = gpu_lib.AdaPMError
    refused(E, lambda: pm.embed(2, t), "worker")
    refused(E, lambda: pm.embed(0, t, 17), "dim")
    refused(E, lambda: pm.embed(0, t, 0), "dim")
    refused(E, lambda: pm.embed(0, t, out=x[:1].expand(6, 16)), "overlap")
    refused(E, lambda: pm.embed(0, t.view(2, 3), out=torch.zeros(80, device="cuda").as_strided((2, 3, 16), (20, 16, 1))),
            "overlap")
    refused(ValueError, lambda: pm.embed(0, t, out=x.double()), "float32")
    refused(ValueError, lambda: pm.embed(0, t, out=x.t().contiguous().t()), "follow")
    refused(ValueError, lambda: pm.embed(0, t, out=x[:5]), "shape")
    refused(ValueError, lambda: pm.embed(0, t.float()), "integers")
    refused(ValueError, lambda: pm.embed(0, t, 8, out=x), "dim")
    refused(E, lambda: pm.embed_grad(5, t, x), "worker")
    refused(E, lambda: pm.embed_grad(0, t, torch.zeros(6, 20, device="cuda")), "dim")
    refused(ValueError, lambda: pm.embed_grad(0, t, x[:5]), "shape")
    refused(ValueError, lambda: pm.embed_grad(0, t, x.double()), "float32")
    g = pm.embed_grad(0, t, x)
    refused(ValueError, lambda: pm.embed_grad(0, torch.cat([t, t]), torch.cat([x, x]), out=g), "out")
    refused(E, lambda: pm.push_grads(2, g.keys, g.rows, 0.1), "worker")
    refused(E, lambda: pm.push_grads(0, g.keys, torch.zeros(6, 17, device="cuda"), 0.1), "dim")
    refused(E, lambda: pm.push_grads(0, g.keys, torch.zeros(6, 6, device="cuda"), 0.1, adagrad=True), "dim")
    refused(ValueError, lambda: pm.push_grads(0, g.keys[:5], g.rows, 0.1), "row")
    refused(ValueError, lambda: pm.push_grads(0, g.keys, g.rows, 0.1, norm=torch.tensor(1.0)), "GPU")
    refused(E, lambda: pm.push_grads(0, g.keys, g.rows, 0.1, norm=torch.ones((), device="cuda"), max_norm=-1.0),
            "negative")
    pm6 = make(gpu_lib, table(20, 12))
    refused(E, lambda: pm6.push_grads(0, g.keys, torch.zeros(6, 6, device="cuda"), 0.1, adagrad=True), "multiple")
    # the C ABI's own checks, behind the binding's
    import ctypes
    lib = gpu_lib.load()
    T = lambda **kw: gpu_lib._Tokens(**{**dict(ids=t.data_ptr(), id_bits=64, has_pad=0, pad=0, outer=1, inner=6,   # noqa: E731
                                               outer_stride=6, inner_stride=1), **kw})
    R = lambda **kw: gpu_lib._Rows(**{**dict(data=x.data_ptr(), type=0, outer_stride=96, inner_stride=16), **kw})  # noqa: E731
    for tok, row in ((T(id_bits=16), R()), (T(), R(type=3)), (T(ids=None), R()), (T(), R(data=None)),
                     (T(outer=2 ** 20, inner=2 ** 20), R()), (T(outer=2 ** 40, inner=2 ** 40), R()),
                     (T(ids=t.data_ptr() + 4), R()), (T(), R(data=x.data_ptr() + 2)), (T(), R(inner_stride=15)),
                     (T(), R(inner_stride=-16))):
        assert lib.adapm_embed(pm._h, 0, ctypes.byref(tok), 16, 1.0, ctypes.byref(row)) == gpu_lib.EINVAL
    host = np.zeros(12, np.int64)
    tok = T(ids=host.ctypes.data, inner_stride=2)
    assert lib.adapm_embed(pm._h, 0, ctypes.byref(tok), 16, 1.0, ctypes.byref(R())) == gpu_lib.EINVAL
    assert lib.adapm_embed(pm._h, 0, None, 16, 1.0, ctypes.byref(R())) == gpu_lib.EINVAL
    assert lib.adapm_embed(None, 0, ctypes.byref(T()), 16, 1.0, ctypes.byref(R())) == gpu_lib.EINVAL
    assert lib.adapm_embed_grad(pm._h, 0, ctypes.byref(T()), 16, 1.0, ctypes.byref(R()), None, None, None) == gpu_lib.EINVAL
    pm.wait()
    assert np.array_equal(pm.read_main(np.arange(20)), table(20, 16))
    pm.close()
    pm6.close()


def test_arrays_between_words_are_refused(gpu_lib):
    pm = make(gpu_lib, table(20, 16))
    t, x = torch.arange(6, device="cuda"), torch.ones(6, 16, device="cuda")
    g = pm.embed_grad(0, t, x)
    pm.wait()
    kept = [a.clone() for a in g]
    import ctypes
    lib = gpu_lib.load()
    tok = gpu_lib._Tokens(t.data_ptr(), 64, 0, 0, 1, 6, 6, 1)
    row = gpu_lib._Rows(x.data_ptr(), 0, 96, 16)
    ptr = [a.data_ptr() for a in g]
    for off in (1, 2, 3):
        for i in range(3):
            at = [p + off * (j == i) for j, p in enumerate(ptr)]
            assert lib.adapm_embed_grad(pm._h, 0, ctypes.byref(tok), 16, 1.0, ctypes.byref(row), *at) == gpu_lib.EINVAL
        for keys, rows in ((ptr[0] + off, ptr[1]), (ptr[0], ptr[1] + off)):
            assert lib.adapm_push_grads(pm._h, 0, keys, rows, 5, 16, 0, 0.1, 0.0, 1.0, 1.0, None) == gpu_lib.EINVAL
        live = gpu_lib._Tensor(ptr[1], 96, ptr[2] + off, 16, 0)
        assert lib.adapm_grad_norm(pm._h, ctypes.byref(live), 1, 1.0, x.data_ptr()) == gpu_lib.EINVAL
    pm.wait()
    assert all(torch.equal(a, b) for a, b in zip(g, kept)) and (x == 1).all()
    assert np.array_equal(pm.read_main(np.arange(20)), table(20, 16))
    pm.close()


def test_a_sort_that_gives_up_leaves_the_outputs(gpu_lib):
    """The bounded wait of a signalled batch's sort runs out (host hook, no GPU fault): ADAPM_ETIMEOUT, nothing written."""
    pm = make(gpu_lib, table(1000, 8))
    n = 20_000
    t = torch.from_numpy(zipf(n, 1000)).cuda()
    pm.intent(0, t, 0, 5)
    g = gpu_lib.RowGrads(torch.full((n,), 7, dtype=torch.int32, device="cuda"), torch.full((n, 8), 5.0, device="cuda"),
                         torch.full((1,), 3, dtype=torch.int32, device="cuda"))
    pm.debug_fail_next_barrier()
    pm.embed_grad(0, t, torch.ones(n, 8, device="cuda"), out=g)
    with pytest.raises(gpu_lib.AdaPMError) as e:
        pm.wait()
    assert e.value.status == gpu_lib.ETIMEOUT
    assert (g.keys == 7).all() and (g.rows == 5.0).all() and int(g.count) == 3
    pm.close()


def test_calls_on_a_stream_of_their_own(gpu_lib):
    """The library's stream is not the caller's: temporaries and results belong to the library's."""
    K, D, n = 3000, 48, 30_000
    init = table(K, D)
    side = torch.cuda.Stream()
    full = torch.from_numpy(zipf(n + 6, K).reshape(6, -1)).cuda()
    grad = torch.randn(6, n // 6, D, device="cuda")
    torch.cuda.synchronize()
    pm = make(gpu_lib, init, stream=side)
    for _ in range(5):   # (freed temporaries would be reused by the next call's on the caller's stream)
        t, short = full[:, :-1], full[:, :-1].to(torch.int16)
        across = grad.transpose(1, 2).contiguous().transpose(1, 2)
        torch.cuda.synchronize()
        out = pm.embed(0, short, scale=2.0)
        g = pm.embed_grad(0, t, across, scale=2.0)
        junk = [torch.full((6, n // 6, D), float("nan"), device="cuda") for _ in range(2)]
        del junk
        side.synchronize()
        assert torch.equal(out.cpu(), torch.from_numpy(init)[t.cpu().to(torch.int16).long()] * 2.0)
        keys, sums, mags, m = plain_grad(t.reshape(-1).cpu().numpy(), grad.reshape(-1, D).double().cpu().numpy(), 2.0)
        check_row_grads(g, keys, sums, 1.01 * (m[:, None] + 1) * U * mags)
    pm.wait()
    pm.close()


@pytest.mark.parametrize("n", [500, 20_000])
def test_recorded_calls_repeat(gpu_lib, n):
    K, D = 900, 16
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        pair = [make(gpu_lib, np.abs(table(K, D)) + 0.1) for _ in range(2)]
        t = torch.from_numpy(zipf(n, K)).cuda()
        x = torch.randn(n, 8, device="cuda")
        more = torch.randn(1000, device="cuda", dtype=torch.bfloat16)
        bufs = [(torch.empty(n, 8, device="cuda"), gpu_lib.RowGrads(
            torch.empty(n, dtype=torch.int32, device="cuda"), torch.zeros(n, 8, device="cuda"),
            torch.empty(1, dtype=torch.int32, device="cuda")), torch.empty((), device="cuda"),
            torch.empty(1000, device="cuda")) for _ in range(2)]
        for pm in pair:
            pm.intent(0, t, 0, 9)

        def calls(pm, b):
            out, g, norm, clipped = b
            pm.embed(0, t, 8, scale=3.0, out=out)
            pm.embed_grad(0, t, x, scale=3.0, out=g)
            pm.grad_norm([g, more], out=norm)
            pm.clip_grads([more], norm, 1.0, out=[clipped])
            pm.push_grads(0, g.keys, g.rows, 0.1, adagrad=True, norm=norm, max_norm=1.0)

        for pm, b in zip(pair, bufs):
            calls(pm, b)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            calls(pair[0], bufs[0])
        for launch in range(3):
            x.normal_()
            t.copy_(torch.from_numpy(zipf(n, K, launch + 50)))
            g.replay()
            calls(pair[1], bufs[1])
            for pm in pair:
                pm.wait()
            u = int(bufs[0][1].count)
            assert u == int(bufs[1][1].count)
            assert torch.equal(bufs[0][0], bufs[1][0]) and torch.equal(bufs[0][1].keys, bufs[1][1].keys)
            assert torch.equal(bufs[0][1].rows[:u], bufs[1][1].rows[:u])
            assert torch.equal(bufs[0][2], bufs[1][2]) and torch.equal(bufs[0][3], bufs[1][3])
            assert np.array_equal(pair[0].read_main(np.arange(K)), pair[1].read_main(np.arange(K)))
            val = [pm.replica_rows(0, np.arange(K)) for pm in pair]
            assert all(np.array_equal(p, q) for p, q in zip(*val))
    for pm in pair:
        pm.close()


def test_offsets_beyond_32_bits(gpu_lib):
    """Store rows, output rows and gradient rows whose element offsets pass 2^32."""
    K, D = 68_000_000, 64                                        # 4.35e9 floats
    pm = gpu_lib.ParameterManager(K, D, 1, replica_capacity=1)
    keys = torch.tensor([1, 5, K // 2, K - 3, K - 1], device="cuda")
    vals = torch.randn(5, D, device="cuda")
    pm.push(0, keys, vals)
    t = keys[torch.tensor([4, 0, 3, 2, 1, 4, 4], device="cuda")].view(1, 7).expand(3, 7)
    buf = torch.empty(3 * 2_200_000_000, dtype=torch.bfloat16, device="cuda")
    out = buf.as_strided((3, 7, D), (2_199_999_992, 136, 1))     # the third sequence begins behind element 2^32
    pm.embed(0, t, scale=0.5, out=out)
    pm.wait()
    want = (vals[[4, 0, 3, 2, 1, 4, 4]] * 0.5).to(torch.bfloat16)
    assert all(torch.equal(out[i], want) for i in range(3))
    g = pm.embed_grad(0, t, out)
    pm.wait()
    assert g.keys[:5].tolist() == keys.tolist()
    x = want.double()
    sums = torch.stack([3 * x[1], 3 * x[4], 3 * x[3], 3 * x[2], 3 * (x[0] + x[5] + x[6])])
    assert ((g.rows[:5].double() - sums).abs() <= 10 * U * sums.abs()).all()
    pm.push_grads(0, g.keys[:5], g.rows[:5], 1.0)
    pm.wait()
    assert torch.allclose(pm.pull(0, keys), vals - g.rows[:5], rtol=1e-6, atol=1e-6)
    pm.close()
