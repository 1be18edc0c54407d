"""The forward pass of the linear layer with outputs that pass the caches by.  Tolerances are
test_gpu_linear's."""
import pytest

from test_gpu_linear import TYPES, Layer, _hc, check_linear

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(4104, 4104, 192), (9000, 2056, 64)])
@pytest.mark.parametrize("dtype", TYPES)
def test_results_past_the_caches(m, n, k, dtype):
    """Outputs of just more than 32 MB, in tiles whole and cut, with the whole epilogue."""
    torch, hc = _hc()
    L = Layer(torch, m, n, k, dtype, 8, 0)
    y, z = torch.empty(m, n, device="cuda", dtype=L.x.dtype), torch.empty(m, n, device="cuda", dtype=L.x.dtype)
    ws = hc.alloc_linear_workspace(L.x, L.w).fill_(0xFF)
    hc.hc_linear(L.x, L.w, y, ws, bias=L.bias, residual=L.residual, z=z, act="gelu", p=0.1, seed=m, draw=n)
    check_linear(torch, L, y, z, "gelu", 0.1, m, n, True, True)
