"""Newton-Schulz orthogonalisation through every way that its products run: tiles of 64, 128 and
256, one and two operand planes, whole, in one group of pieces, in two, or as whole rounds and
pieces; the apply's first, middle and last step, with and without a rest in smaller tiles; either
orientation; batches.  The formula is taken in 64 bits on the GPU.

Tolerances, in the 2-norm relative to the result.  fp32: 1e-5 up to five steps, 2e-6 a step after
(operands of 22 bits and fp32 sums).  bf16: the result's rounding is 2^-9 at most.  With two
operand planes (a shorter side of at most 256) nothing but the fp32 forms' error is added.  With
one, a model of the roundings (fp16 operands, X as an operand and an fp16 rest) adds, before the
result is rounded, on random matrices 4e-4 after three steps, 1.3e-3 after four, 2.1e-3 after five,
2.4e-3 after six and 3.4e-3 after nine: 3.5e-4 a step is allowed on top of the rounding.  On
matrices of low rank over noise it adds 5.7e-4 to 7.3e-4 after five steps, 1.3e-2 to 1.6e-2 without
the rest of X: 3e-3 in all tells the two apart."""
import pytest

pytestmark = pytest.mark.gpu

MUON = (3.4445, -4.7750, 2.0315)
LOWRANK_ONE_PLANE = 3e-3


def _hc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2402_07529_amd as hc
    return torch, hc


def _formula(torch, x, steps, coeffs=MUON, eps=1e-7, scale=1.0):
    """[batch, m, n] in 64 bits."""
    x = x.double()
    wide = x.shape[1] <= x.shape[2]
    y = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + eps)
    y = y if wide else y.transpose(1, 2).contiguous()
    for t in range(steps):
        a, b, c = coeffs if isinstance(coeffs[0], float) else coeffs[t]
        g = torch.bmm(y, y.transpose(1, 2).contiguous())
        y = a * y + torch.bmm(b * g + c * torch.bmm(g, g), y)
    return (y if wide else y.transpose(1, 2)) * scale


def _off(torch, got, want):
    """The largest of the matrices' relative errors."""
    d = torch.linalg.vector_norm(got.double() - want, dim=(1, 2))
    return float((d / torch.linalg.vector_norm(want, dim=(1, 2))).max())


def _matrices(torch, batch, m, n, kind, dtype, gap=0, pad=0):
    """Matrices in one flat buffer of NaN, at a stride of m rows of n + pad and gap elements more."""
    gen = torch.Generator(device="cuda").manual_seed(31 * m + n)
    ld, stride = n + pad, m * (n + pad) + gap
    flat = torch.full((1 + batch * stride,), float("nan"), device="cuda", dtype=getattr(torch, dtype))
    x = flat.as_strided((batch, m, n), (stride, ld, 1), 1)
    for b in range(batch):
        y = torch.randn(m, n, device="cuda", generator=gen)
        if kind == "lowrank":
            r = max(1, min(m, n) // 8)
            y = 0.05 * y + torch.randn(m, r, device="cuda", generator=gen) @ torch.randn(r, n, device="cuda", generator=gen)
        x[b] = y * (b + 1)
    return x


def _run(torch, hc, x, **kw):
    """The result, written into a layout like x's, after a check that nothing else was."""
    flat = torch.full((1 + x.shape[0] * x.stride(0) + x.shape[1] * x.stride(1),), 7.0, device="cuda", dtype=x.dtype)
    out = flat.as_strided(x.shape, x.stride(), 1)
    ws = hc.alloc_orthogonalise_workspace(x)
    ws.fill_(255)                                   # NaNs: it is not read before it is written
    hc.hc_orthogonalise(x, out, ws, **kw)
    got = out.clone()
    out.fill_(7.0)
    assert bool((flat == 7.0).all()), "wrote outside its matrices"
    return got


def _tolerance(dtype, m, n, steps):
    fp32 = 1e-5 * max(1.0, steps / 5)
    if dtype == "float32":
        return fp32
    return 2.0**-9 + (fp32 if min(m, n) <= 256 else 3.5e-4 * steps)


PLANS = [  # what the products of each run as, by their sizes
    # one plane (bf16, a shorter side above 256)
    ("bfloat16", 2, 300, 520, 1001, 1),     # all in 64-tiles
    ("bfloat16", 2, 520, 300, 7, 0),
    ("bfloat16", 16, 307, 493, 3, 2),
    ("bfloat16", 2, 300, 1500, 0, 0),       # Gram: 64-tiles in one group of pieces
    ("bfloat16", 24, 300, 14000, 0, 0),     # Gram: 64-tiles in two groups
    ("bfloat16", 12, 768, 768, 5000, 0),    # apply: 128-tiles
    ("bfloat16", 2, 268, 9418, 0, 0),       # Gram in pieces, apply in 128-tiles
    ("bfloat16", 1, 1800, 4600, 0, 0),      # Gram: 128-tiles in pieces; apply: 128-tiles, the rest in 64
    ("bfloat16", 1, 4600, 1800, 0, 0),
    ("bfloat16", 12, 640, 10000, 0, 0),     # Gram: 128-tiles in two groups
    ("bfloat16", 48, 400, 400, 9, 0),       # Gram, square: 128-tiles; apply: 256-tiles
    ("bfloat16", 48, 400, 768, 0, 0),       # apply: 256-tiles, the rest in 128
    ("bfloat16", 5, 7000, 400, 11, 0),      # apply: 256-tiles, the rest in 64
    ("bfloat16", 5, 900, 8192, 0, 0),       # Gram: 256-tiles in one group of pieces
    ("bfloat16", 16, 900, 900, 0, 0),       # all in 256-tiles
    ("bfloat16", 16, 900, 2700, 0, 0),      # Gram: whole rounds of 128-tiles and pieces; square: 256-tiles
    ("bfloat16", 5, 2500, 2500, 0, 0),      # Gram, square: whole rounds of 256-tiles and pieces
    ("bfloat16", 2, 2700, 2700, 0, 0),      # Gram, square: 128-tiles; apply: 256-tiles
    ("bfloat16", 1, 9000, 4000, 0, 0),      # tall; apply: 256-tiles, the rest in 128
    ("bfloat16", 1, 4096, 25088, 0, 0),     # Gram: 256-tiles in two groups; square: whole rounds and pieces
    ("bfloat16", 1, 24576, 4000, 0, 0),
    # two planes
    ("bfloat16", 12, 200, 2700, 5, 0),      # Gram: 64-tiles in pieces; apply: 256-tiles
    ("bfloat16", 12, 2700, 200, 0, 3),
    ("bfloat16", 12, 200, 5500, 0, 0),      # apply: 256-tiles, the rest in 64
    ("bfloat16", 100, 200, 768, 0, 0),      # apply: 256-tiles, the rest in 128
    ("bfloat16", 48, 130, 10000, 0, 0),     # Gram: 64-tiles in two groups
    ("float32", 35, 223, 950, 0, 0),        # apply: 256-tiles
    ("float32", 24, 384, 900, 13, 1),       # apply: 128-tiles, the rest in 64
    ("float32", 12, 768, 768, 0, 0),        # all in 128-tiles
    ("float32", 157, 403, 510, 0, 0),       # Gram, square: 256-tiles
    ("float32", 5, 900, 4600, 0, 0),        # Gram: 128-tiles in two groups
    ("float32", 16, 900, 900, 0, 0),        # Gram, square: whole rounds of 128-tiles and pieces
    ("float32", 2, 1500, 1500, 0, 0),       # Gram, square: 128-tiles in pieces
    ("float32", 1, 640, 640, 0, 0),         # Gram, square: 64-tiles in pieces
    ("float32", 1, 6000, 1500, 0, 0),       # tall; apply: 128-tiles, the rest in 64
    # a shorter side of at most 128: several slabs a workgroup, parts summed by a launch or read by all
    ("float32", 10, 40, 5000, 7, 0),
    ("float32", 9, 100, 4000, 0, 1),
    ("bfloat16", 9, 4000, 100, 0, 0),
    ("float32", 300, 40, 128, 0, 0),
    ("bfloat16", 600, 128, 70, 3, 0),
]


@pytest.mark.parametrize("dtype,batch,m,n,gap,pad", PLANS)
def test_against_formula(dtype, batch, m, n, gap, pad):
    torch, hc = _hc()
    x = _matrices(torch, batch, m, n, "lowrank", dtype, gap, pad)
    got = _run(torch, hc, x, scale=-0.75)
    tol = LOWRANK_ONE_PLANE if dtype == "bfloat16" and min(m, n) > 256 else _tolerance(dtype, m, n, 5)
    assert _off(torch, got, _formula(torch, x, 5, scale=-0.75)) <= tol


STEPS = [(1, 300, 520), (1, 520, 300), (1, 640, 384), (3, 400, 900), (48, 400, 400), (2, 150, 200)]


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 4, 6, 9])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("batch,m,n", STEPS)
def test_steps_and_scale(steps, dtype, batch, m, n):
    """One step is the first and the last at once."""
    torch, hc = _hc()
    x = _matrices(torch, batch, m, n, "random", dtype, gap=5)
    got = _run(torch, hc, x, steps=steps, scale=-0.25)
    assert _off(torch, got, _formula(torch, x, steps, scale=-0.25)) <= _tolerance(dtype, m, n, steps)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("batch,m,n", [(1, 300, 520), (2, 640, 384)])
def test_coefficients_per_step(dtype, batch, m, n):
    """Other powers of two for the operands in every step.  The schedule's slopes (2, 3.4, then at most
    1.5) are below those of as many default steps."""
    torch, hc = _hc()
    x = _matrices(torch, batch, m, n, "random", dtype)
    schedule = [(2.0, -1.5, 0.5), MUON] + [(1.5, -0.5, 0.0)] * 4
    got = _run(torch, hc, x, steps=6, coeffs=schedule, scale=0.2)
    assert _off(torch, got, _formula(torch, x, 6, schedule, scale=0.2)) <= _tolerance(dtype, m, n, 6)


@pytest.mark.parametrize("m,n", [(300, 400), (400, 300)])
def test_zero_nan_and_infinity_in_one_plane(m, n):
    """A zero matrix stays zero; NaN or infinity takes its own matrix and no other."""
    torch, hc = _hc()
    x = _matrices(torch, 6, m, n, "random", "bfloat16")
    x[0] = 0
    x[1, 3, 4], x[3, 0, 0], x[5, m - 1, n - 1] = float("nan"), float("inf"), float("-inf")
    got = _run(torch, hc, x)
    assert not bool(got[0].any())
    for b in (1, 3, 5):
        assert bool(got[b].isnan().all()), b
    good = x[2:5:2]
    assert _off(torch, got[2:5:2], _formula(torch, good, 5)) <= _tolerance("bfloat16", m, n, 5)


@pytest.mark.parametrize("dtype,batch,m,n", [("bfloat16", 1, 300, 520), ("bfloat16", 2, 300, 1500),
                                             ("bfloat16", 12, 768, 768), ("float32", 1, 640, 640),
                                             ("float32", 10, 40, 5000)])
def test_repeats_and_graph_replays(dtype, batch, m, n):
    torch, hc = _hc()
    x = _matrices(torch, batch, m, n, "random", dtype)
    x = x.contiguous()
    out, want = torch.empty_like(x), torch.empty_like(x)
    ws = hc.alloc_orthogonalise_workspace(x)
    hc.hc_orthogonalise(x, want, ws)
    hc.hc_orthogonalise(x, out, ws)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hc.hc_orthogonalise(x, out, ws)
    for k in range(4):
        x.mul_(-1.5).add_(0.125 * k)
        graph.replay()
        torch.cuda.synchronize()
        hc.hc_orthogonalise(x, want, ws)
        assert torch.equal(out, want), k
