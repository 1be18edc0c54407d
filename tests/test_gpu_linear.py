"""The linear layer and its gradient against their definition in 64 bits.

Tolerances, from the arithmetic.  A sum of t products in fp32, in any grouping, is within (t + 2)
2^-24 of the sum S of its terms' magnitudes (products of 16-bit values are exact; fp32 in two fp16
parts is 2^-22 off, and a product of two leaves the rests' out: 3 2^-22; below 2^-29 of a row's largest
2^-51 of that).  An activation's slope is at most 1.13, and its own
error is layer_reference.FUNCTION relative to its factors.  Dropout's factor and a residual are 3
roundings.  The result is rounded by half a unit.  In the gradient of 16-bit types dz is rounded by
half a unit h before the products; where the gradient is wider bf16 takes three parts (2^-24) and
fp16 two (2^-22).  What fp16 holds below its normal range is 2^-25 off, as a rest in units of 2^-11
2^-36."""
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
SLOPE = 1.13
PARTS, FAR = 3 * 2.0**-22, 2.0**-50   # FAR: 2^-51 of either side


def _hc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2402_07529_amd as hc
    return torch, hc


class Layer:
    """Inputs of a layer on the device, with `gap` elements between rows that start `offset` in."""

    def __init__(self, torch, m, n, k, dtype, gap=0, offset=0, seed=0, dz=1.0):
        gen = torch.Generator().manual_seed(seed * 1000003 + m * 31 + n * 7 + k)
        self.dtype, dt = dtype, getattr(torch, dtype)

        def make(rows, cols, std):
            flat = torch.full((offset + rows * (cols + gap) + 8,), float("nan"), device="cuda", dtype=dt)
            view = flat.as_strided((rows, cols), (cols + gap, 1), offset)
            return view.copy_(torch.randn(rows, cols, generator=gen) * std)

        self.x, self.w = make(m, k, 1.0), make(n, k, k**-0.5)
        self.bias = (torch.randn(n, generator=gen) * 0.5).to(dt).cuda()
        self.residual, self.z, self.dy = make(m, n, 1.0), make(m, n, 1.5), make(m, n, dz)


def _out(torch, rows, cols, gap, offset, dtype):
    flat = torch.full((offset + rows * (cols + gap) + 8,), 7, device="cuda").to(dtype)
    return flat, flat.as_strided((rows, cols), (cols + gap, 1), offset)


def _untouched(torch, flat, view, offset):
    """Everything but the view still holds 7."""
    view.fill_(7)
    return bool((flat == 7).all())


def _within(got, want, tol, what):
    off = (got.cpu().double() - want).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), float((off - tol).max()))


def _f(torch, m, n, p, seed, draw):
    return torch.from_numpy(ref.factors(m, n, p, seed, draw)) if p else torch.ones(m, n, dtype=torch.float64)


def check_linear(torch, L, got_y, got_z, act, p, seed, draw, bias, residual):
    d = L.dtype
    x, w = L.x.cpu().double(), L.w.cpu().double()
    k = x.shape[1]
    z = x @ w.t()
    off = (x.abs() @ w.abs().t()) * ((k + 2) * ref.UNIT + (PARTS if d == "float32" else 0))
    if d == "float32":
        off += k * FAR * x.abs().amax(1)[:, None] * w.abs().amax(1)[None, :]
    if bias:
        b = L.bias.cpu().double()
        z, off = z + b, off + 2 * ref.UNIT * (z.abs() + b.abs())
    if got_z is not None:
        _within(got_z, z, off + ref.HALF[d] * (z.abs() + off) + ref.FLOOR[d], "z")
    a, _ = ref.activate(torch, act, z)
    size = z.abs() if act in ("gelu", "silu") else torch.ones_like(z)
    off = SLOPE * off + (0 if act in ("none", "relu") else ref.FUNCTION[d] * size)
    f = _f(torch, z.shape[0], z.shape[1], p, seed, draw)
    y = a * f
    off = off * f + 3 * ref.UNIT * y.abs()
    if residual:
        r = L.residual.cpu().double()
        y, off = y + r, off + 3 * ref.UNIT * (y.abs() + r.abs())
    _within(got_y, y, off + ref.HALF[d] * (y.abs() + off) + ref.FLOOR[d], "y")


def check_grad(torch, L, act, p, seed, draw, dx, dw, db, out, old=None, fixed=None):
    """old: what dw and db held before (accumulate)."""
    d, h = L.dtype, ref.HALF[L.dtype]
    dy, z, x, w = (t.cpu().double() for t in (L.dy, L.z, L.x, L.w))
    m, n = dy.shape
    f = _f(torch, m, n, p, seed, draw)
    dz = dy * f
    slope_off = 3 * ref.UNIT * dz.abs()
    if act != "none":
        _, slope = ref.activate(torch, act, z)
        size = 1 + (z.abs() if act in ("gelu", "silu") else 0)
        slope_off = slope_off * SLOPE + dz.abs() * size * (0 if act == "relu" else 2 * ref.FUNCTION[d])
        dz = dz * slope
    plain = act == "none" and not p
    part = PARTS if d == "float32" else 0
    one = slope_off if plain or d == "float32" else slope_off + h * dz.abs() + ref.FLOOR[d]
    if dx is not None:
        want, size = dz @ w, dz.abs() @ w.abs()
        off = one @ w.abs() + size * ((n + 2) * ref.UNIT + part) * (1 + h)
        if d == "float32":
            off += n * FAR * dz.abs().amax(1)[:, None] * w.abs().amax(0)[None, :]
        _within(dx, want, off + h * (want.abs() + off) + ref.FLOOR[d], "dx")

    def widened(want, off, name, got):
        base = old[name].cpu().double() if old else torch.zeros_like(want)
        if fixed:
            off = off * fixed + 0.5 + 2 * ref.UNIT * (want.abs() * fixed)
            want = (want * fixed + base).clamp(-2**31 + 1, 2**31 - 1)
            _within(got, want, off, name)
            return
        off = off + 2 * ref.UNIT * (want.abs() + base.abs()) if old else off
        want = want + base
        _within(got, want, off + ref.HALF[out] * (want.abs() + off) + ref.FLOOR[out], name)

    if dw is not None:
        two = plain or d == "float32"
        wide, terms = one, m
        if not two and out not in ("bfloat16", "float16"):
            wide = slope_off + h * h * dz.abs() * (1 if d == "float16" else h) + ref.FLOOR[d] * 2**-11
            terms = (2 if d == "float16" else 3) * m
        want, size = dz.t() @ x, dz.abs().t() @ x.abs()
        off = wide.t() @ x.abs() + size * ((terms + 2) * ref.UNIT + part) * (1 + h)
        if d == "float32":
            off += m * FAR * dz.abs().amax(0)[:, None] * x.abs().amax(0)[None, :]
        widened(want, off, "dw", dw)
    if db is not None:
        widened(dz.sum(0), slope_off.sum(0) + dz.abs().sum(0) * (m + 2) * ref.UNIT, "db", db)


SHAPES = [(1, 1, 1), (1, 768, 768), (16, 768, 768), (3, 5, 7), (64, 64, 64), (65, 63, 33), (700, 150, 1500),
          (33, 1000, 129), (257, 96, 64), (130, 520, 264), (512, 256, 512), (100, 77, 3000), (2, 4099, 40),
          (2049, 24, 16), (300, 320, 1000)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap,offset", [(0, 0), (3, 1), (8, 8)])
def test_linear(m, n, k, dtype, gap, offset):
    torch, hc = _hc()
    dt = getattr(torch, dtype)
    L = Layer(torch, m, n, k, dtype, gap, offset)
    ws = hc.alloc_linear_workspace(L.x, L.w)
    for act, p, bias, residual, wants_z in (("none", 0.0, False, False, False), ("gelu", 0.1, True, True, True),
                                            ("relu", 0.5, True, False, False)):
        fy, y = _out(torch, m, n, gap, offset, dt)
        fz, z = _out(torch, m, n, gap, offset, dt)
        ws.fill_(0xFF)
        hc.hc_linear(L.x, L.w, y, ws, bias=L.bias if bias else None, residual=L.residual if residual else None,
                     z=z if wants_z else None, act=act, p=p, seed=99 + m, draw=(3 << 32) + n)
        check_linear(torch, L, y, z if wants_z else None, act, p, 99 + m, (3 << 32) + n, bias, residual)
        assert _untouched(torch, fy, y, offset) and _untouched(torch, fz, z, offset)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu", "tanh", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES)
def test_activations(act, dtype):
    torch, hc = _hc()
    L = Layer(torch, 70, 90, 50, dtype, seed=3)
    L.w.mul_(3.0)
    y, z = torch.empty_like(L.z), torch.empty_like(L.z)
    hc.hc_linear(L.x, L.w, y, hc.alloc_linear_workspace(L.x, L.w), bias=L.bias, z=z, act=act)
    check_linear(torch, L, y, z, act, 0.0, 0, 0, True, False)
    dx, dw, db = torch.empty_like(L.x), torch.empty_like(L.w), torch.empty_like(L.bias)
    hc.hc_linear_grad(L.dy, hc.alloc_linear_grad_workspace(L.x, L.w), x=L.x, w=L.w, z=L.z, dx=dx, dw=dw, db=db,
                      act=act)
    check_grad(torch, L, act, 0.0, 0, 0, dx, dw, db, dtype)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu", "tanh", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES)
def test_activations_far_out(act, dtype):
    """One input, weight 1: the activation at single values.  Tails go to their limits, NaN stays."""
    torch, hc = _hc()
    inf = float("inf")
    z = torch.tensor([[0.0, -0.0, 1e-3, -1e-3, 3.0, -3.0, 9.0, -9.0, 30.0, -30.0, 1e4, -1e4, inf, -inf,
                       float("nan")]], device="cuda").to(getattr(torch, dtype)).t().contiguous()
    w, y, dz, dx = torch.ones(1, 1, device="cuda", dtype=z.dtype), torch.empty_like(z), torch.ones_like(z), \
        torch.empty_like(z)
    hc.hc_linear(z, w, y, hc.alloc_linear_workspace(z, w), act=act)
    hc.hc_linear_grad(dz, hc.alloc_linear_grad_workspace(z, w), w=w, z=z, dx=dx, act=act)
    limits = {"relu": (inf, 0), "gelu": (inf, 0), "silu": (inf, 0), "tanh": (1, -1), "sigmoid": (1, 0)}[act]
    assert (float(y[12]), float(y[13])) == limits and bool(torch.isnan(y[14]).all())
    ends = {"relu": 1, "gelu": 1, "silu": 1, "tanh": 0, "sigmoid": 0}[act]
    assert (float(dx[12]), float(dx[13])) == (ends, 0) and bool(torch.isnan(dx[14]).all())
    v = z[:12].cpu().double()
    a, slope = ref.activate(torch, act, v)
    size = v.abs() if act in ("gelu", "silu") else torch.ones_like(v)
    tol = ref.FUNCTION[dtype] * size.clamp(max=40) + ref.HALF[dtype] * a.abs() + ref.FLOOR[dtype] + 2.0**-126
    _within(y[:12], a, tol, "y")
    # slopes of size 1 + |z|, times phi or s' below 2^-24 past |z| of 17
    tol = 2 * ref.FUNCTION[dtype] * (1 + size.clamp(max=17)) + 2 * ref.HALF[dtype] * slope.abs() \
        + 2 * ref.FLOOR[dtype] + 2.0**-126
    _within(dx[:12], slope, tol, "dx")


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap,offset", [(0, 0), (3, 1), (8, 8)])
def test_gradient(m, n, k, dtype, gap, offset):
    torch, hc = _hc()
    dt = getattr(torch, dtype)
    L = Layer(torch, m, n, k, dtype, gap, offset)
    ws = hc.alloc_linear_grad_workspace(L.x, L.w)
    for act, p, out in (("none", 0.0, "float32"), ("gelu", 0.1, dtype), ("relu", 0.5, "float32"),
                        ("silu", 0.0, "bfloat16")):
        wide = getattr(torch, out)
        fx, dx = _out(torch, m, k, gap, offset, dt)
        fw, dw = _out(torch, n, k, gap, offset, wide)
        db = torch.empty(n, device="cuda", dtype=wide)
        ws.fill_(0xFF)
        hc.hc_linear_grad(L.dy, ws, x=L.x, w=L.w, z=L.z if act != "none" else None, dx=dx, dw=dw, db=db, act=act, p=p,
                          seed=5, draw=m)
        check_grad(torch, L, act, p, 5, m, dx, dw, db, out)
        assert _untouched(torch, fx, dx, offset) and _untouched(torch, fw, dw, offset)


@pytest.mark.parametrize("dtype", TYPES)
def test_each_gradient_alone(dtype):
    torch, hc = _hc()
    L = Layer(torch, 200, 100, 72, dtype)
    ws = hc.alloc_linear_grad_workspace(L.x, L.w)

    def outs():
        return torch.empty_like(L.x), torch.empty_like(L.w), torch.empty_like(L.bias)

    dx, dw, db = outs()
    hc.hc_linear_grad(L.dy, ws, x=L.x, w=L.w, z=L.z, dx=dx, dw=dw, db=db, act="tanh", p=0.2, seed=1)
    ax, aw, ab = outs()
    hc.hc_linear_grad(L.dy, ws, w=L.w, z=L.z, dx=ax, act="tanh", p=0.2, seed=1)
    hc.hc_linear_grad(L.dy, ws, x=L.x, z=L.z, dw=aw, act="tanh", p=0.2, seed=1)
    hc.hc_linear_grad(L.dy, ws, z=L.z, db=ab, act="tanh", p=0.2, seed=1)
    assert torch.equal(dx, ax) and torch.equal(dw, aw) and torch.equal(db, ab)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("out", ["float32", "bfloat16", "float16"])
def test_accumulate(dtype, out):
    torch, hc = _hc()
    L = Layer(torch, 300, 130, 70, dtype)
    ws = hc.alloc_linear_grad_workspace(L.x, L.w)
    dw, db = (torch.randn(130, 70, device="cuda").to(getattr(torch, out)),
              torch.randn(130, device="cuda").to(getattr(torch, out)))
    old = dict(dw=dw.clone(), db=db.clone())
    hc.hc_linear_grad(L.dy, ws, x=L.x, z=L.z, dw=dw, db=db, act="sigmoid", accumulate=True)
    check_grad(torch, L, "sigmoid", 0.0, 0, 0, None, dw, db, out, old)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_fixed_point(dtype, accumulate):
    torch, hc = _hc()
    L = Layer(torch, 150, 60, 90, dtype, dz=1e-2)
    ws = hc.alloc_linear_grad_workspace(L.x, L.w)
    dw = torch.randint(-1000, 1000, (60, 90), device="cuda", dtype=torch.int32)
    db = torch.randint(-1000, 1000, (60,), device="cuda", dtype=torch.int32)
    old = dict(dw=dw.clone(), db=db.clone()) if accumulate else None
    hc.hc_linear_grad(L.dy, ws, x=L.x, z=L.z, dw=dw, db=db, act="gelu", p=0.3, seed=4, fixed=2.0**20,
                      accumulate=accumulate)
    check_grad(torch, L, "gelu", 0.3, 4, 0, None, dw, db, "int32", old, fixed=2.0**20)


def test_fixed_point_saturates():
    torch, hc = _hc()
    top = 2**31 - 1
    x = torch.ones(4, 3, device="cuda")
    dy = torch.tensor([[3e6, -3e6, float("nan"), 1.0]], device="cuda").expand(4, 4).contiguous()
    ws = hc.alloc_linear_grad_workspace(x, torch.empty(4, 3, device="cuda"))
    dw = torch.full((4, 3), 5, device="cuda", dtype=torch.int32)
    db = torch.full((4,), 5, device="cuda", dtype=torch.int32)
    for accumulate in (False, True, True):
        hc.hc_linear_grad(dy, ws, x=x, dw=dw, db=db, fixed=2.0**20, accumulate=accumulate)
    want = torch.tensor([top, -top, 0, 3 * 4 * 2**20], dtype=torch.int32)
    assert torch.equal(db.cpu(), want) and torch.equal(dw.cpu(), want[:, None].expand(4, 3))


def test_gradient_against_differences():
    """dL/dtheta of L = sum(y * c) by central differences of the forward pass in fp32: a difference
    of step e is off by e^2 / 6 of the third derivative and 2^-24 |y c| sqrt(mn) / e."""
    torch, hc = _hc()
    m, n, k, e = 6, 5, 4, 2.0**-6
    L = Layer(torch, m, n, k, "float32", seed=8)
    c = torch.randn(m, n, device="cuda")
    ws = hc.alloc_linear_workspace(L.x, L.w)
    y, z = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    kw = dict(act="gelu", p=0.4, seed=3, draw=1)

    def loss():
        hc.hc_linear(L.x, L.w, y, ws, bias=L.bias, residual=L.residual, z=z, **kw)
        return float((y.double() * c.double()).sum())

    loss()
    dx, dw, db = torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
    hc.hc_linear_grad(c, hc.alloc_linear_grad_workspace(L.x, L.w), x=L.x, w=L.w, z=z, dx=dx, dw=dw, db=db, **kw)
    for t, g in ((L.x, dx), (L.w, dw), (L.bias, db)):
        for at in range(t.numel()):
            v = t.reshape(-1)[at].item()
            t.view(-1)[at] = v + e
            up = loss()
            t.view(-1)[at] = v - e
            down = loss()
            t.view(-1)[at] = v
            # third derivatives of gelu are below 1.6; inputs and weights below 4 in size
            scale = float(c.abs().sum()) / 0.6
            tol = e * e / 6 * 1.6 * scale * 4**3 / 8 + 2**-22 * scale * 4 / e
            assert abs((up - down) / (2 * e) - g.reshape(-1)[at].item()) < tol


def test_mask_is_dropouts():
    torch, hc = _hc()
    L = Layer(torch, 130, 77, 40, "float32")
    ws = hc.alloc_linear_workspace(L.x, L.w)
    a, b, c = (torch.empty(130, 77, device="cuda") for _ in range(3))
    hc.hc_linear(L.x, L.w, a, ws, bias=L.bias, act="silu", p=0.3, seed=12, draw=34, residual=L.residual)
    hc.hc_linear(L.x, L.w, b, ws, bias=L.bias, act="silu")
    hc.hc_dropout(b, c, 0.3, 12, 34, residual=L.residual)
    assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", TYPES)
def test_residual_in_place_and_three_dimensions(dtype):
    torch, hc = _hc()
    dt = getattr(torch, dtype)
    x, w = torch.randn(4, 9, 56, device="cuda").to(dt), torch.randn(40, 56, device="cuda").to(dt)
    r = torch.randn(4, 9, 40, device="cuda").to(dt)
    ws, y = hc.alloc_linear_workspace(x, w), torch.empty_like(r)
    hc.hc_linear(x, w, y, ws, residual=r, p=0.1, seed=1)
    hc.hc_linear(x, w, r, ws, residual=r, p=0.1, seed=1)
    assert torch.equal(y, r)


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_stays_in_its_row_or_column(dtype):
    torch, hc = _hc()
    L = Layer(torch, 90, 80, 70, dtype)
    L.x[13, 5] = float("nan")
    L.w[21, 6] = float("inf")
    y = torch.empty_like(L.z)
    hc.hc_linear(L.x, L.w, y, hc.alloc_linear_workspace(L.x, L.w))
    bad = ~torch.isfinite(y.cpu())
    want = torch.zeros(90, 80, dtype=torch.bool)
    want[13], want[:, 21] = True, True
    assert torch.equal(bad, want)
    # dropped rows of the output gradient leave nothing, whatever they hold
    f = torch.from_numpy(ref.factors(90, 80, 0.5, 6, 7)).cuda()
    dy = torch.randn(90, 80, device="cuda").to(L.x.dtype)
    clean = torch.where(f == 0, 0.0, dy)
    dy[f == 0] = float("nan")
    ws = hc.alloc_linear_grad_workspace(L.x, L.w)
    L.x[13, 5], L.w[21, 6] = 1.0, 1.0
    for g, outs in ((dy, []), (clean, [])):
        dx, dw, db = torch.empty_like(L.x), torch.empty_like(L.w), torch.empty_like(L.bias)
        hc.hc_linear_grad(g, ws, x=L.x, w=L.w, dx=dx, dw=dw, db=db, p=0.5, seed=6, draw=7)
        outs += [dx, dw, db]
        if g is clean:
            assert all(torch.equal(a, b) for a, b in zip(first, outs))
        first = outs


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(dtype):
    torch, hc = _hc()
    dt = getattr(torch, dtype)
    x, w = torch.empty(0, 24, device="cuda", dtype=dt), torch.randn(16, 24, device="cuda").to(dt)
    y = torch.empty(0, 16, device="cuda", dtype=dt)
    hc.hc_linear(x, w, y, hc.alloc_linear_workspace(x, w))
    ws = hc.alloc_linear_grad_workspace(x, w)
    dw, db = torch.full((16, 24), 3.0, device="cuda"), torch.full((16,), 3.0, device="cuda")
    hc.hc_linear_grad(y, ws, x=x, w=w, dx=x.clone(), dw=dw, db=db, accumulate=True)
    assert bool((dw == 3).all()) and bool((db == 3).all())
    hc.hc_linear_grad(y, ws, x=x, w=w, dx=x.clone(), dw=dw, db=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_two_calls_agree_bit_for_bit_and_fewer_rows_fit(dtype):
    torch, hc = _hc()
    L = Layer(torch, 600, 200, 300, dtype)
    ws, gws = hc.alloc_linear_workspace(L.x, L.w), hc.alloc_linear_grad_workspace(L.x, L.w)
    for m in (600, 599, 333, 64, 5, 1):
        x, dy, z = L.x[:m], L.dy[:m], L.z[:m]
        got = []
        for _ in range(2):
            y, dx, dw, db = (torch.empty_like(dy), torch.empty_like(x), torch.empty_like(L.w),
                             torch.empty_like(L.bias))
            hc.hc_linear(x, L.w, y, ws, bias=L.bias, act="gelu", p=0.1, seed=1)
            hc.hc_linear_grad(dy, gws, x=x, w=L.w, z=z, dx=dx, dw=dw, db=db, act="gelu", p=0.1, seed=1)
            got.append((y, dx, dw, db))
        assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_run_together_captured_and_replayed():
    """Two layers forward and back with one dropout between, as a training step uses them, in a graph
    whose counter goes on, against the eager calls at that draw."""
    torch, hc = _hc()
    m, n, k = 257, 72, 136
    dt, dev = torch.bfloat16, "cuda"
    x, w1, w2 = (torch.randn(m, k, device=dev).to(dt), (torch.randn(n, k, device=dev) * 0.1).to(dt),
                 (torch.randn(k, n, device=dev) * 0.1).to(dt))
    b1, b2 = torch.randn(n, device=dev).to(dt), torch.randn(k, device=dev).to(dt)
    dy = torch.randn(m, k, device=dev).to(dt)
    wf = [hc.alloc_linear_workspace(x, w1), hc.alloc_linear_workspace(dy.new_empty(m, n), w2)]
    wg = [hc.alloc_linear_grad_workspace(x, w1), hc.alloc_linear_grad_workspace(dy.new_empty(m, n), w2)]

    def bufs():
        return dict(z=x.new_empty(m, n), h=x.new_empty(m, n), y=x.new_empty(m, k), d=x.new_empty(m, k),
                    dh=x.new_empty(m, n), dx=x.new_empty(m, k), dw1=torch.empty(n, k, device=dev),
                    dw2=torch.empty(k, n, device=dev), db1=torch.empty(n, device=dev),
                    db2=torch.empty(k, device=dev))

    def step(b, draw, counter=None):
        hc.hc_linear(x, w1, b["h"], wf[0], bias=b1, z=b["z"], act="gelu", p=0.1, seed=4, draw=draw, counter=counter)
        hc.hc_linear(b["h"], w2, b["y"], wf[1], bias=b2, residual=x)
        hc.hc_dropout(b["y"], b["y"], 0.2, 5, draw, counter=counter)
        hc.hc_dropout(dy, b["d"], 0.2, 5, draw, counter=counter)
        hc.hc_linear_grad(b["d"], wg[1], x=b["h"], w=w2, dx=b["dh"], dw=b["dw2"], db=b["db2"])
        hc.hc_linear_grad(b["dh"], wg[0], x=x, w=w1, z=b["z"], dx=b["dx"], dw=b["dw1"], db=b["db1"], act="gelu",
                          p=0.1, seed=4, draw=draw, counter=counter)

    counter, got, want = torch.zeros(1, device=dev, dtype=torch.int64), bufs(), bufs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(got, 0, counter)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(got, 0, counter)
            counter.add_(1)
    torch.cuda.synchronize()
    counter.zero_()
    for i in range(3):
        for b in got.values():
            b.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        step(want, i)
        for name in got:
            assert torch.equal(got[name], want[name]), (i, name)


def test_offsets_past_32_bits():
    torch, hc = _hc()
    m, k, n = 2**20 + 5, 4100, 8                     # 4.3e9 elements of x
    x = torch.zeros(m, k, device="cuda", dtype=torch.bfloat16)
    at = [0, 1047552, m - 1]
    w = (torch.randn(n, k, device="cuda") * k**-0.5).bfloat16()
    rows = torch.randn(3, k, device="cuda").bfloat16()
    x[at] = rows
    y = torch.empty(m, n, device="cuda", dtype=torch.bfloat16)
    hc.hc_linear(x, w, y, hc.alloc_linear_workspace(x, w))
    want = rows.cpu().double() @ w.cpu().double().t()
    tol = (rows.cpu().double().abs() @ w.cpu().double().abs().t()) * (k + 2) * ref.UNIT
    _within(y[at], want, tol + 2**-8 * (want.abs() + tol), "y")
    assert int((y != 0).any(1).sum()) == 3
    dy = torch.zeros(m, n, device="cuda", dtype=torch.bfloat16)
    dy[at] = torch.randn(3, n, device="cuda").bfloat16()
    dw = torch.empty(n, k, device="cuda")
    hc.hc_linear_grad(dy, hc.alloc_linear_grad_workspace(x, w), x=x, dw=dw)
    a, b = dy[at].cpu().double(), rows.cpu().double()
    _within(dw, a.t() @ b, (a.abs().t() @ b.abs()) * 5 * ref.UNIT, "dw")


def test_refusals():
    torch, hc = _hc()
    x, w, y = (torch.randn(6, 8, device="cuda"), torch.randn(5, 8, device="cuda"),
               torch.empty(6, 5, device="cuda"))
    ws, gws = hc.alloc_linear_workspace(x, w), hc.alloc_linear_grad_workspace(x, w)
    for kw in (dict(x=x.cpu()), dict(w=w[:, :7]), dict(y=y[:5]), dict(y=y.bfloat16()), dict(w=w.half()),
               dict(bias=torch.zeros(4, device="cuda")), dict(bias=torch.zeros(5, device="cuda").bfloat16()),
               dict(residual=torch.zeros(6, 4, device="cuda")), dict(z=torch.zeros(5, 5, device="cuda")),
               dict(act="swish"), dict(x=x.int(), w=w.int(), y=y.int())):
        a = dict(x=x, w=w, y=y, ws=ws)
        a.update(kw)
        with pytest.raises((ValueError, hc.HCError)):
            hc.hc_linear(**a)
    dy, dw = torch.randn(6, 5, device="cuda"), torch.empty(5, 8, device="cuda")
    for kw in (dict(dx=x.clone()), dict(dw=dw, x=None), dict(act="relu", dw=dw), dict(dw=dw[:4]),
               dict(dw=dw, db=torch.empty(5, device="cuda", dtype=torch.int32)), dict(dw=dw.double()),
               dict(db=torch.empty(4, device="cuda"))):
        a = dict(dy=dy, ws=gws, x=x)
        a.update(kw)
        with pytest.raises((ValueError, hc.HCError)):
            hc.hc_linear_grad(**a)
    with pytest.raises(hc.HCError):
        hc.hc_linear(x, w, y, ws, p=1.01)
    big = torch.randn(600, 64, device="cuda")
    with pytest.raises(hc.HCError):
        hc.hc_linear(big, big, torch.empty(600, 600, device="cuda"), ws[:256])


# sizes that take each of the tiles: 256 (whole ones, cut ones, a ragged edge), 128 and 64
TILED = [(2100, 1000, 520), (4096, 4096, 192), (1030, 2056, 72), (520, 264, 4104), (8200, 264, 136), (333, 520, 1000)]


@pytest.mark.parametrize("m,n,k", TILED)
@pytest.mark.parametrize("dtype", TYPES)
def test_tiles(m, n, k, dtype):
    torch, hc = _hc()
    dt = getattr(torch, dtype)
    L = Layer(torch, m, n, k, dtype, 8, 8)
    y, z = torch.empty(m, n, device="cuda", dtype=dt), torch.empty(m, n, device="cuda", dtype=dt)
    ws = hc.alloc_linear_workspace(L.x, L.w).fill_(0xFF)
    hc.hc_linear(L.x, L.w, y, ws, bias=L.bias, residual=L.residual, z=z, act="gelu", p=0.1, seed=m, draw=n)
    check_linear(torch, L, y, z, "gelu", 0.1, m, n, True, True)
    for act, p, out in (("none", 0.0, "float32"), ("silu", 0.1, "float32"), ("gelu", 0.1, dtype)):
        wide = getattr(torch, out)
        dx, dw, db = torch.empty(m, k, device="cuda", dtype=dt), torch.empty(n, k, device="cuda", dtype=wide), \
            torch.empty(n, device="cuda", dtype=wide)
        ws = hc.alloc_linear_grad_workspace(L.x, L.w).fill_(0xFF)
        hc.hc_linear_grad(L.dy, ws, x=L.x, w=L.w, z=L.z, dx=dx, dw=dw, db=db, act=act, p=p, seed=m, draw=n)
        check_grad(torch, L, act, p, m, n, dx, dw, db, out)


def test_fp32_rows_and_columns_of_far_sizes():
    """Rows and columns between 1e-30 and 1e30: fp32 products in parts keep their accuracy in each."""
    torch, hc = _hc()
    m, n, k = 1100, 1000, 1300
    gen = torch.Generator().manual_seed(5)

    def sizes(count):
        return 10.0 ** torch.randint(-15, 16, (count,), generator=gen).float()

    L = Layer(torch, m, n, k, "float32")
    L.x.mul_(sizes(m)[:, None].cuda())
    L.w.mul_(sizes(n)[:, None].cuda())
    y = torch.empty(m, n, device="cuda")
    hc.hc_linear(L.x, L.w, y, hc.alloc_linear_workspace(L.x, L.w))
    L.bias.zero_()
    check_linear(torch, L, y, None, "none", 0.0, 0, 0, False, False)
    # dx sees rows of dy and columns of w, dw columns of dy and of x
    L = Layer(torch, m, n, k, "float32")
    dx, dw = torch.empty_like(L.x), torch.empty_like(L.w)
    ws = hc.alloc_linear_grad_workspace(L.x, L.w)
    L.dy.mul_(sizes(m)[:, None].cuda())
    L.w.mul_(sizes(k)[None, :].cuda())
    hc.hc_linear_grad(L.dy, ws, w=L.w, dx=dx)
    check_grad(torch, L, "none", 0.0, 0, 0, dx, None, None, "float32")
    L.dy.copy_(torch.randn(m, n, generator=gen)).mul_(sizes(n)[None, :].cuda())
    L.x.mul_(sizes(k)[None, :].cuda())
    hc.hc_linear_grad(L.dy, ws, x=L.x, dw=dw)
    check_grad(torch, L, "none", 0.0, 0, 0, None, dw, None, "float32")


def test_fp32_zeros_subnormals_and_nan_in_parts():
    torch, hc = _hc()
    m, n, k = 1100, 1000, 1300
    L = Layer(torch, m, n, k, "float32")
    L.x[3] = 0
    L.x[4] = 2.0**-149
    L.x[5, 7] = float("nan")
    L.w[6] = 0
    L.w[8] = 3.0e38
    y = torch.empty(m, n, device="cuda")
    hc.hc_linear(L.x, L.w, y, hc.alloc_linear_workspace(L.x, L.w))
    y = y.cpu()
    assert bool((y[3, :6] == 0).all()) and bool(torch.isnan(y[5]).all())
    rest = torch.cat([y[:5], y[6:]])
    assert bool((rest[:, 6] == 0).all()) and not bool(torch.isnan(rest).any())
    want = L.x[:3].cpu().double().sum(1) * float(L.w[8, 0])
    tol = L.x[:3].cpu().double().abs().sum(1) * 3.0e38 * ((k + 2) * ref.UNIT + PARTS)
    inside = want.abs() + tol < 3.4e38
    assert bool(((rest[:3, 8].double() - want).abs() <= tol)[inside].all())


@pytest.mark.parametrize("m,n,k", [(16384, 64, 128), (20001, 40, 24), (33000, 7, 250), (17000, 64, 256)])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_through_a_small_matrix(m, n, k, dtype):
    torch, hc = _hc()
    dt = getattr(torch, dtype)
    for (a, b), gap in (((n, k), 0), ((k, n), 3)):   # the forward pass's and dx's
        L = Layer(torch, m, a, b, dtype, gap)
        y, dx = torch.empty(m, a, device="cuda", dtype=dt), torch.empty(m, b, device="cuda", dtype=dt)
        hc.hc_linear(L.x, L.w, y, hc.alloc_linear_workspace(L.x, L.w), bias=L.bias, residual=L.residual, act="silu",
                     p=0.1, seed=m)
        check_linear(torch, L, y, None, "silu", 0.1, m, 0, True, True)
        hc.hc_linear_grad(L.dy, hc.alloc_linear_grad_workspace(L.x, L.w), w=L.w, dx=dx)
        check_grad(torch, L, "none", 0.0, 0, 0, dx, None, None, dtype)


@pytest.mark.parametrize("dtype,act", [("float32", "none"), ("float32", "gelu"), ("bfloat16", "gelu"), ("float16", "silu")])
def test_large_gradients_captured_replayed_and_on_two_streams(dtype, act):
    """Packed, cut and joined products in a graph, against eager calls, and two calls at once."""
    torch, hc = _hc()
    m, n, k = 1100, 1000, 1300
    L = [Layer(torch, m, n, k, dtype, seed=s) for s in (1, 2)]
    p = 0.0 if act == "none" else 0.2

    def outs():
        dt = L[0].x.dtype
        return [torch.full((m, k), 9.0, device="cuda", dtype=dt), torch.full((n, k), 9.0, device="cuda"),
                torch.full((n,), 9.0, device="cuda"), torch.full((m, n), 9.0, device="cuda", dtype=dt)]

    ws = [(hc.alloc_linear_workspace(l.x, l.w), hc.alloc_linear_grad_workspace(l.x, l.w)) for l in L]

    def run(i, o):
        l = L[i]
        hc.hc_linear(l.x, l.w, o[3], ws[i][0], bias=l.bias, residual=l.residual, act=act, p=p, seed=i)
        hc.hc_linear_grad(l.dy, ws[i][1], x=l.x, w=l.w, z=l.z, dx=o[0], dw=o[1], db=o[2], act=act, p=p, seed=i)

    want = [outs(), outs()]
    for i in (0, 1):
        run(i, want[i])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [outs(), outs()]
    torch.cuda.synchronize()
    for i in (0, 1, 0, 1):
        with torch.cuda.stream(streams[i]):
            run(i, got[i])
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))
    graph, o = torch.cuda.CUDAGraph(), outs()
    with torch.cuda.graph(graph, stream=streams[0]):
        run(0, o)
    for _ in range(3):
        for t in o:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o, want[0]))
        L[0].dy.mul_(1.0)          # eager work between the replays
        torch.cuda.synchronize()
