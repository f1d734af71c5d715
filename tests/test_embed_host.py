"""Host logic of the token-embedding calls: how strides become two levels, and refusals that need no GPU."""
import itertools

import numpy as np
import pytest
import torch

from paper_2206_00470_gb300 import adapm
from paper_2206_00470_gb300 import build as libbuild


def offsets(shape, strides):
    return np.array([sum(i * s for i, s in zip(at, strides)) for at in itertools.product(*map(range, shape))],
                    dtype=np.int64)


def levels(got, i):
    outer, inner, *steps = got
    return (np.arange(outer)[:, None] * steps[i][0] + np.arange(inner) * steps[i][1]).reshape(-1)


VIEWS = [
    lambda b: b, lambda b: b[:, :-1], lambda b: b[1:, ::2], lambda b: b.t(), lambda b: b[2], lambda b: b[:, 3],
    lambda b: b[1:2, :4], lambda b: b[:1, :1], lambda b: b[0, 0], lambda b: b[:3].expand(3, 12),
    lambda b: b[:1].expand(5, 12), lambda b: b[:, :1].expand(6, 4), lambda b: b.reshape(6, 3, 4),
    lambda b: b.reshape(6, 3, 4).transpose(0, 1), lambda b: b.reshape(6, 3, 4)[:, :, :2], lambda b: b[:, :0],
    lambda b: b.reshape(2, 3, 12)[:, 1:], lambda b: b.reshape(2, 3, 3, 4)[:, :, :1], lambda b: b.reshape(1, 6, 1, 12),
]


@pytest.mark.parametrize("view", range(len(VIEWS)))
@pytest.mark.parametrize("rows", range(3))
def test_two_levels_reach_the_same_elements(view, rows):
    tokens = VIEWS[view](torch.arange(72).reshape(6, 12))
    wide = [torch.empty((*tokens.shape, 5)), torch.empty((*tokens.shape, 9))[..., :5],
            torch.empty((*reversed(tokens.shape), 5)).permute(*reversed(range(tokens.dim())), tokens.dim())][rows]
    assert wide.shape[:-1] == tokens.shape
    got = adapm._two_levels(tokens.shape, tokens.stride(), wide.stride()[:-1])
    if got is None:   # (more than two steps: the call copies)
        assert tokens.dim() >= 3
        return
    assert got[0] * got[1] == tokens.numel()
    if tokens.numel():
        assert np.array_equal(levels(got, 0), offsets(tokens.shape, tokens.stride()))
        assert np.array_equal(levels(got, 1), offsets(tokens.shape, wide.stride()[:-1]))


def test_lists_refuse_what_is_not_on_the_gpu():
    with pytest.raises(ValueError):
        adapm.GradList([torch.zeros(4)])
    assert adapm.GradList([]).n == 0


def test_norms_are_gpu_scalars():
    with pytest.raises(ValueError):
        adapm._check_norm(torch.zeros(()))
    adapm._check_norm(None)


class Recorder:
    """Stands for the library: every call is noted and answered with ADAPM_OK."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or adapm.OK


@pytest.fixture
def manager():
    """The binding's half of a manager."""
    pm = adapm.ParameterManager.__new__(adapm.ParameterManager)
    pm._lib, pm._h, pm.D = Recorder(), None, 8
    pm._t, pm._r = adapm._Tokens(), adapm._Rows()
    pm._t_ref, pm._r_ref = adapm.ctypes.byref(pm._t), adapm.ctypes.byref(pm._r)
    return pm


@pytest.mark.parametrize("out", [torch.zeros((), dtype=torch.float16), torch.zeros(3, dtype=torch.bfloat16)[1],
                                 torch.zeros((), dtype=torch.float64), torch.zeros((), dtype=torch.int32),
                                 torch.zeros(2), torch.zeros(0), torch.zeros(8, dtype=torch.uint8)[1]])
def test_a_norm_goes_into_one_float(manager, out):
    with pytest.raises(ValueError):
        manager.grad_norm([], out=out)
    assert not manager._lib.calls
    for fits in (torch.zeros(()), torch.zeros(5)[3], torch.zeros(1, 1)):
        assert manager.grad_norm([], out=fits) is fits
        assert manager._lib.calls.pop()[1][-1] == fits.data_ptr()


def test_types():
    assert [adapm._type_of(t) for t in (torch.float32, torch.float16, torch.bfloat16)] == [0, 1, 2]
    with pytest.raises(ValueError):
        adapm._type_of(torch.float64)


def test_entry_points_refuse_a_null_context():
    lib = adapm.load(libbuild.build())
    assert lib.adapm_embed(None, 0, None, 1, 1.0, None) == adapm.EINVAL
    assert lib.adapm_embed_grad(None, 0, None, 1, 1.0, None, None, None, None) == adapm.EINVAL
    assert lib.adapm_grad_norm(None, None, 0, 1.0, None) == adapm.EINVAL
    assert lib.adapm_clip_grads(None, None, None, 0, 1.0, 1.0, None) == adapm.EINVAL
    assert lib.adapm_push_grads(None, 0, None, None, 0, 4, 0, 0.1, 0.0, 1.0, 1.0, None) == adapm.EINVAL
