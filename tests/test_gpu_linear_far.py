"""Dense layers at the ends of their ranges: numbers whose squares leave fp32."""
import pytest
import torch

from .test_gpu_linear import ACTS, check, check_grad

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pm(gpu_lib):
    pm = gpu_lib.ParameterManager(4, 4, 1)
    yield pm
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
