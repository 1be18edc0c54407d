"""Gradients in fixed point, and added to what is there, by every way that a product goes: small, direct
and in tiles of each size, whole, cut and joined.  Tolerances are test_gpu_linear's; an added result is
one more sum, a fixed-point one is off by half a unit more."""
import pytest

from test_gpu_linear import TYPES, Layer, _hc, check_grad

pytestmark = pytest.mark.gpu

# dw in 16 bits (rows apart by a multiple of 8 | of 11): tiles of 128 whole | direct; tiles of 64 cut |
# direct and joined; direct and joined; direct | direct; tiles of 128 whole and cut; tiles of 256 whole;
# tiles of 128 in many pieces; small.  fp32: direct, joined, and in planes whole and cut
SHAPES = [(192, 2048, 2048, 8), (192, 2048, 2048, 11), (1030, 1000, 520, 8), (1030, 1000, 520, 11),
          (1100, 1000, 1300, 0), (700, 1500, 1500, 0), (1088, 2056, 4104, 0), (512, 4096, 4096, 0),
          (16384, 768, 768, 0), (24, 520, 1048, 0)]


@pytest.mark.parametrize("m,n,k,gap", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_types_written_and_added(m, n, k, gap, dtype):
    torch, hc = _hc()
    L = Layer(torch, m, n, k, dtype, gap, dz=1e-2)
    ws = hc.alloc_linear_grad_workspace(L.x, L.w).fill_(0xFF)
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    for out, accumulate, act, p in (("int32", False, "gelu", 0.1), ("int32", True, "none", 0.0),
                                    ("float32", True, "silu", 0.5), (dtype, True, "gelu", 0.1)):
        def start(*shape):
            if out == "int32":
                return torch.randint(-2**20, 2**20, shape, device="cuda", dtype=torch.int32, generator=gen)
            return torch.randn(*shape, device="cuda", generator=gen).to(getattr(torch, out))

        flat = start(n * (k + gap) + 5)
        before = flat.clone()
        at = 5 if gap == 11 else 0
        dw, db = flat.as_strided((n, k), (k + gap, 1), at), start(n)
        old = dict(dw=dw.clone(), db=db.clone()) if accumulate else None
        hc.hc_linear_grad(L.dy, ws, x=L.x, z=L.z if act != "none" else None, dw=dw, db=db, act=act, p=p, seed=6,
                          draw=m, fixed=2.0**20, accumulate=accumulate)
        check_grad(torch, L, act, p, 6, m, None, dw, db, out, old, fixed=2.0**20 if out == "int32" else None)
        dw.copy_(before.as_strided((n, k), (k + gap, 1), at))
        assert torch.equal(flat, before), "wrote outside its rows"


@pytest.mark.parametrize("m,n,k", [(192, 2048, 2048), (1030, 1000, 520), (512, 4096, 4096)])
@pytest.mark.parametrize("dtype", TYPES)
def test_large_fixed_point_saturates(m, n, k, dtype):
    """Sums past 2^31 units and sums with NaN in them, written and added."""
    torch, hc = _hc()
    top, dt = 2**31 - 1, getattr(torch, dtype)
    x, dy = torch.ones(m, k, device="cuda", dtype=dt), torch.zeros(m, n, device="cuda", dtype=dt)
    dy[:, 0], dy[:, 1], dy[0, 2], dy[:, n - 1] = 2.0**14, -2.0**14, float("nan"), 1.0
    ws = hc.alloc_linear_grad_workspace(x, torch.empty(n, k, device="cuda", dtype=dt))
    dw = torch.full((n, k), 5, device="cuda", dtype=torch.int32)
    db = torch.full((n,), 5, device="cuda", dtype=torch.int32)
    want = torch.zeros(n, device="cuda", dtype=torch.int64)
    want[0], want[1], want[n - 1] = top, -top, m * 2**10
    for accumulate, base in ((False, 0), (True, 1), (True, 2)):
        hc.hc_linear_grad(dy, ws, x=x, dw=dw, db=db, fixed=2.0**10, accumulate=accumulate)
        now = (want * (base + 1)).clamp(-top, top).int()
        assert torch.equal(db, now) and torch.equal(dw, now[:, None].expand(n, k))
