"""The binding of the linear layer refuses a bias or its gradient that is not n elements long."""
import pytest

from test_gpu_linear import TYPES, _hc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count", [1, 4, 6, 40])
def test_a_bias_of_another_length_is_refused(dtype, count):
    torch, hc = _hc()
    dt = getattr(torch, dtype)
    x, w, y = (torch.ones(s, device="cuda", dtype=dt) for s in ((6, 8), (5, 8), (6, 5)))
    bias = torch.ones(count, device="cuda", dtype=dt)
    with pytest.raises(ValueError, match="bias must be 5 contiguous elements"):
        hc.hc_linear(x, w, y, hc.alloc_linear_workspace(x, w), bias=bias)
    ws, dw = hc.alloc_linear_grad_workspace(x, w), torch.empty(5, 8, device="cuda", dtype=dt)
    for kw in (dict(), dict(x=x, dw=dw)):
        with pytest.raises(ValueError, match="db must be 5 contiguous elements"):
            hc.hc_linear_grad(y, ws, db=bias, **kw)


def test_a_bias_of_two_dimensions_is_taken():
    torch, hc = _hc()
    x, w, y = (torch.ones(s, device="cuda") for s in ((6, 8), (5, 8), (6, 5)))
    bias = torch.arange(5.0, device="cuda")
    hc.hc_linear(x, w, y, hc.alloc_linear_workspace(x, w), bias=bias[None, :])
    assert torch.equal(y, 8 + bias.expand(6, 5))
