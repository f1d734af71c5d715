"""Host logic of the calls on dense layers: refusals that need no GPU, and what the binding hands to the library."""
import ctypes

import pytest
import torch

from paper_2206_00470_gb300 import adapm
from paper_2206_00470_gb300 import build as libbuild


class Recorder:
    """Stands for the library: every call is noted and answered with ADAPM_OK."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or adapm.OK


@pytest.fixture
def manager():
    """The binding's half of a manager, which takes CPU tensors for its own device's."""
    pm = adapm.ParameterManager.__new__(adapm.ParameterManager)
    pm._lib, pm._h, pm.D = Recorder(), None, 8
    pm._d, pm._device, pm._index, pm._handle = adapm._Dense(), torch.device("cpu"), -1, 0
    pm._on_stream = lambda: adapm._NOTHING
    adapm._type_of(torch.float32)
    return pm


def test_entry_points_refuse_a_null_context():
    lib = adapm.load(libbuild.build())
    assert lib.adapm_layer_norm(None, None, None, None, None, 1e-5, None, None) == adapm.EINVAL
    assert lib.adapm_layer_norm_grad(None, None, None, None, None, None, None, None, None) == adapm.EINVAL
    assert lib.adapm_linear(None, None, None, None, None, 0, None, None, None) == adapm.EINVAL
    assert lib.adapm_linear_grad(None, None, None, None, None, None, 0, None, None, None) == adapm.EINVAL
    assert lib.adapm_distill(None, None, None, None, 1.0, 1.0, None, 0.0, 1.0, None, None, None) == adapm.EINVAL


def test_tensors_of_another_device_are_refused(manager):
    manager._index = 0
    x, w = torch.zeros(3, 8), torch.zeros(8, 4)
    for call in (lambda: manager.layer_norm(x, out=x), lambda: manager.layer_norm_grad(x, x, torch.zeros(3, 2), out=adapm.NormGrads(x, None, None)),
                 lambda: manager.linear(x, w, out=torch.zeros(3, 4)), lambda: manager.distill(x, loss=torch.zeros(3)),
                 lambda: manager.linear_grad(x, w, torch.zeros(3, 4), out=adapm.LinearGrads(x, w, None))):
        with pytest.raises(ValueError):
            call()
    assert not manager._lib.calls


@pytest.mark.parametrize("view,outer,inner,steps", [
    (lambda t: t, 1, 30, (0, 8)), (lambda t: t[:, :-1], 5, 5, (48, 8)), (lambda t: t.transpose(0, 1), 6, 5, (8, 48)),
    (lambda t: t[..., :6], 1, 30, (0, 8)), (lambda t: t[2], 1, 6, (0, 8)), (lambda t: t[1, 1], 1, 1, (0, 8)),
    (lambda t: t[:0], 1, 0, (0, 8)), (lambda t: t[:, :1].expand(5, 4, 8), 5, 4, (48, 0))])
def test_rows_are_described_where_they_lie(manager, view, outer, inner, steps):
    x = view(torch.arange(240.0).view(5, 6, 8))
    out = torch.empty(x.shape)
    manager.layer_norm(x, out=out)
    s, r = manager._d.shape, manager._d.rows[0]
    assert s.dim == x.shape[-1] and s.outer * s.inner == outer * inner and r.data == (x.data_ptr() or None)
    at = [r.outer_stride * o + r.inner_stride * i for o in range(s.outer) for i in range(s.inner)]
    want = [sum(i * n for i, n in zip(index, x.stride())) for index in torch.cartesian_prod(
        *(torch.arange(n) for n in x.shape[:-1])).view(-1, max(1, x.dim() - 1)).tolist()] if x.dim() > 1 and x.numel() else at
    assert at == want


def test_matrices_keep_their_strides(manager):
    x, w = torch.zeros(7, 16, dtype=torch.half)[:, :8], torch.zeros(4, 8, dtype=torch.half).t()
    manager.linear(x, w, out=torch.zeros(7, 4, dtype=torch.half))
    m = manager._d.matrices
    assert (m[0].row_stride, m[0].col_stride, m[1].row_stride, m[1].col_stride) == (16, 1, 1, 8)
    layer = manager._d.layer
    assert (layer.rows, layer.ins, layer.outs) == (7, 8, 4)
    # rows that are not one step apart are copied, outputs of such rows refused
    wide = torch.zeros(3, 5, 8, dtype=torch.half)[:, :4]
    manager.linear(wide, w, out=torch.zeros(3, 4, 4, dtype=torch.half))
    assert m[0].row_stride == 8 and m[0].data != wide.data_ptr()
    with pytest.raises(ValueError):
        manager.linear(torch.zeros(3, 4, 8, dtype=torch.half), w, out=torch.zeros(3, 5, 4, dtype=torch.half)[:, :4])


def test_activations_by_name(manager):
    assert [adapm._activation(a) for a in (None, "none", "relu", "gelu", "gelu_tanh", "silu", "tanh")] == [0, 0, 1, 2, 3, 4, 5]
    with pytest.raises(ValueError):
        adapm._activation("sigmoid")
    header = open(libbuild.INCLUDE + "/adapm.h").read()
    for name, value in adapm.ACTIVATIONS.items():
        assert f"#define ADAPM_ACTIVATION_{(name or 'none').upper()} {value}\n" in header


def test_optional_arrays_are_null(manager):
    x, w = torch.zeros(3, 8, dtype=torch.half), torch.zeros(8, 4, dtype=torch.half)
    manager.linear(x, w, out=torch.zeros(3, 4, dtype=torch.half))
    assert [manager._lib.calls[-1][1][i] for i in (4, 6, 8)] == [None, None, None]
    manager.layer_norm(x, out=x)
    assert [manager._lib.calls[-1][1][i] for i in (3, 4, 7)] == [None, None, None]
    manager.distill(x, loss=torch.zeros(3))
    assert [manager._lib.calls[-1][1][i] for i in (3, 6, 9, 10)] == [None, None, None, None]


def test_labels_take_any_pad(manager):
    x, y = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int32)
    for pad, has in ((None, 0), (-100, 1), (2 ** 70, 0), (2 ** 63 - 1, 1)):
        manager.distill(x, labels=y, hard=1.0, pad=pad, loss=torch.zeros(3))
        assert manager._d.labels.has_pad == has and manager._d.labels.id_bits == 32
        assert not has or manager._d.labels.pad == pad


def test_structures_have_the_size_of_the_header():
    """As a C compiler lays them out: the fields in order, naturally aligned."""
    assert [ctypes.sizeof(t) for t in (adapm._Shape, adapm._Vector, adapm._Matrix, adapm._Layer, adapm._Teacher,
                                       adapm._Labels)] == [24, 16, 32, 16, 32, 24]
