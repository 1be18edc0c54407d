"""The linear layer's gradient at the ends of fp16, output gradients near its largest and smallest values; and
what stands in places that dropout drops.

fp16: dz is held in units of 2^e, the smallest power of two no less than dropout's scale times the largest
slope (1.13 for gelu and silu, else 1), at least 1.  So none overflows, and what fp16 holds below its normal
range is 2^(e - 25) off, in a high part and a rest 2^(e - 36).  All else is test_gpu_linear's."""
import math

import pytest

import layer_reference as ref
from test_gpu_linear import SLOPE, TYPES, Layer, _f, _hc, _within

pytestmark = pytest.mark.gpu


def _unit(act, p):
    scale = 65536.0 / (65536 - ref.limit(p)) if p else 1.0
    return 2.0 ** max(0, math.ceil(math.log2(scale * (SLOPE if act in ("gelu", "silu") else 1.0))))


def _check(torch, L, act, p, seed, draw, dx, dw, db, out, fixed=1.0):
    """db: or None."""
    h, least = ref.HALF["float16"], ref.FLOOR["float16"]
    dy, z, x, w = (t.cpu().double() for t in (L.dy, L.z, L.x, L.w))
    m, n = dy.shape
    dz = dy * _f(torch, m, n, p, seed, draw)
    off = 3 * ref.UNIT * dz.abs()
    if act != "none":
        _, slope = ref.activate(torch, act, z)
        size = 1 + (z.abs() if act in ("gelu", "silu") else 0)
        off = off * SLOPE + dz.abs() * size * (0 if act == "relu" else 2 * ref.FUNCTION["float16"])
        dz = dz * slope
    one = off + h * dz.abs() + least * _unit(act, p)
    wide = off + h * h * dz.abs() + least * _unit(act, p) * 2**-11
    want = dz @ w
    tol = one @ w.abs() + (dz.abs() @ w.abs()) * (n + 2) * ref.UNIT * (1 + h)
    _within(dx, want, tol + h * (want.abs() + tol) + least, "dx")

    def check(got, want, tol, name):
        if out == "int32":
            _within(got, want * fixed, tol * fixed + 0.5 + 2 * ref.UNIT * want.abs() * fixed, name)
        else:
            _within(got, want, tol + ref.HALF[out] * (want.abs() + tol) + ref.FLOOR[out], name)

    want, each = dz.t() @ x, one if out == "float16" else wide
    check(dw, want, each.t() @ x.abs() + (dz.abs().t() @ x.abs()) * (2 * m + 2) * ref.UNIT * (1 + h), "dw")
    if db is not None:
        check(db, dz.sum(0), off.sum(0) + dz.abs().sum(0) * (m + 2) * ref.UNIT, "db")


def _run(torch, hc, L, act, p, out, fixed, wants_db=True):
    m, n, k = L.dy.shape[0], L.dy.shape[1], L.x.shape[1]
    dt = getattr(torch, out)
    dx, dw = torch.empty_like(L.x), torch.empty(n, k, device="cuda", dtype=dt)
    db = torch.empty(n, device="cuda", dtype=dt) if wants_db else None
    ws = hc.alloc_linear_grad_workspace(L.x, L.w).fill_(0xFF)
    hc.hc_linear_grad(L.dy, ws, x=L.x, w=L.w, z=L.z if act != "none" else None, dx=dx, dw=dw, db=db, act=act, p=p,
                      seed=4, draw=n, fixed=fixed)
    _check(torch, L, act, p, 4, n, dx, dw, db, out, fixed)


# small, direct, direct and joined, in tiles whole and cut, copied
SHAPES = [(150, 60, 90), (700, 150, 1500), (1030, 1000, 520), (200, 2048, 2048), (1100, 1000, 1300)]
HOW = [("none", 0.5), ("gelu", 0.0), ("silu", 0.5), ("relu", 0.9), ("tanh", 0.1)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("act,p", HOW)
@pytest.mark.parametrize("out", ["float32", "int32", "float16"])
def test_fp16_output_gradients_near_the_largest(m, n, k, act, p, out):
    torch, hc = _hc()
    L = Layer(torch, m, n, k, "float16", seed=2)
    gen = torch.Generator().manual_seed(m)
    big = 65504 * (0.4 + 0.6 * torch.rand(m, n, generator=gen)) * (torch.randint(0, 2, (m, n), generator=gen) * 2 - 1)
    L.dy.copy_(torch.where(torch.rand(m, n, generator=gen) < 0.2, big, torch.randn(m, n, generator=gen)))
    L.dy[0, 0] = 65504
    # results that their types hold, and zeros, which an infinite dz would make NaN
    L.w.mul_(2.0**-8)
    if out == "float16":
        L.x.mul_(2.0**-10)
    L.x[:, 3] = 0
    L.x[::5] = 0
    L.w[::7] = 0
    _run(torch, hc, L, act, p, out, 16.0, wants_db=out != "float16")


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("act,p", HOW)
@pytest.mark.parametrize("out", ["float32", "float16"])
def test_fp16_output_gradients_near_the_smallest(m, n, k, act, p, out):
    torch, hc = _hc()
    L = Layer(torch, m, n, k, "float16", seed=5)
    sizes = 2.0 ** -torch.randint(8, 25, (m, n), generator=torch.Generator().manual_seed(n)).float()
    L.dy.mul_(sizes.cuda())
    _run(torch, hc, L, act, p, out, 1.0)


@pytest.mark.parametrize("m,n,k", [(90, 80, 70), (1030, 1000, 520)])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu", "tanh", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_dropped_element_has_no_gradient_whatever_z_holds(m, n, k, act, dtype):
    torch, hc = _hc()
    L = Layer(torch, m, n, k, dtype, seed=6)
    dropped = (torch.from_numpy(ref.factors(m, n, 0.5, 8, 9)) == 0).cuda()
    ws = hc.alloc_linear_grad_workspace(L.x, L.w)

    def grads(z):
        dx, dw = torch.empty_like(L.x), torch.empty(n, k, device="cuda")
        db = torch.empty(n, device="cuda")
        hc.hc_linear_grad(L.dy, ws, x=L.x, w=L.w, z=z, dx=dx, dw=dw, db=db, act=act, p=0.5, seed=8, draw=9)
        return dx, dw, db

    want = grads(L.z)
    for bad in (float("nan"), float("inf"), float("-inf")):
        got = grads(torch.where(dropped, bad, L.z))
        assert all(torch.equal(a, b) for a, b in zip(got, want)), bad
    # one that is kept stays: in its row of dx and dw, and in db
    i, j = (int(v) for v in (~dropped).nonzero()[37])
    z = L.z.clone()
    z[i, j] = float("nan")
    dx, dw, db = grads(z)
    for t, rows in ((dx, i), (dw, j), (db, j)):
        bad = torch.isnan(t).reshape(t.shape[0], -1)
        assert bool(bad[rows].all()) and int(bad.any(1).sum()) == 1
