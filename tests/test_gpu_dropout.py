"""Dropout against its definition, with masks from a generator written apart.

Tolerance, from the arithmetic: a kept element is one fp32 product with a factor rounded to fp32, a
residual one more sum: 3 half-units of 2^-24 of the terms' magnitudes, plus half a unit of the type."""
import numpy as np
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu


def _hc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2402_07529_amd as hc
    return torch, hc


def _strided(torch, rows, cols, gap, offset, dtype, gen=None):
    flat = torch.full((offset + rows * (cols + gap) + 8,), 7, device="cuda", dtype=dtype)
    view = flat.as_strided((rows, cols), (cols + gap, 1), offset)
    if gen is not None:
        view.copy_(torch.randn(rows, cols, generator=gen))
    return flat, view


def _check(torch, got, x, residual, f, dtype):
    want, size = x * f, (x * f).abs()
    if residual is not None:
        want, size = want + residual, size + residual.abs()
    tol = 3 * ref.UNIT * size + ref.HALF[dtype] * want.abs() * (1 + 2**-10) + ref.FLOOR[dtype]
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), float((off - tol).max())


SHAPES = [(1, 1), (1, 8), (3, 7), (700, 1500), (33, 768), (5, 9), (1000, 1), (257, 13), (2, 4099), (64, 512),
          (1, 100003), (4096, 24)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("gap,offset", [(0, 0), (3, 1)])
def test_dropout(rows, cols, dtype, gap, offset):
    torch, hc = _hc()
    gen = torch.Generator().manual_seed(rows * 31 + cols)
    dt = getattr(torch, dtype)
    seed, draw = 0xDEADBEEF12345678 + rows, (7 << 33) + cols
    _, x = _strided(torch, rows, cols, gap, offset, dt, gen)
    _, residual = _strided(torch, rows, cols, gap + 2, offset, dt, gen)
    for p in (0.1, 0.5, 0.65):
        f = torch.from_numpy(ref.factors(rows, cols, p, seed, draw))
        for r in (None, residual):
            flat, out = _strided(torch, rows, cols, gap, offset, dt)
            before = flat.clone()
            hc.hc_dropout(x, out, p, seed, draw, residual=r)
            _check(torch, out.cpu(), x.cpu().double(), None if r is None else r.cpu().double(), f, dtype)
            out.copy_(before.as_strided(out.shape, out.stride(), offset))
            assert torch.equal(flat, before), "wrote outside its rows"


def test_edges_of_p():
    torch, hc = _hc()
    x = torch.randn(9, 21, device="cuda")
    x[0, 0], x[1, 1] = float("nan"), float("inf")
    out = torch.empty_like(x)
    for p in (0.0, 2.0**-18):      # nothing is dropped
        hc.hc_dropout(x, out, p, 5)
        assert torch.equal(out.nan_to_num(), x.nan_to_num())
    for p in (1.0, 1.0 - 2.0**-18):  # everything is, whatever it holds
        hc.hc_dropout(x, out, p, 5)
        assert torch.equal(out, torch.zeros_like(x))
    r = torch.randn(9, 21, device="cuda")
    hc.hc_dropout(x, out, 1.0, 5, residual=r)
    assert torch.equal(out, r)


def test_dropped_infinities_and_nan_leave_nothing():
    torch, hc = _hc()
    rows, cols, p = 40, 50, 0.5
    f = torch.from_numpy(ref.factors(rows, cols, p, 11, 3)).cuda()
    x = torch.randn(rows, cols, device="cuda").bfloat16()
    x[f == 0] = float("nan")
    x[:, 7][f[:, 7] == 0] = float("-inf")
    r = torch.randn(rows, cols, device="cuda").bfloat16()
    out = torch.empty_like(x)
    hc.hc_dropout(x, out, p, 11, 3, residual=r)
    assert bool(torch.isfinite(out).all())
    assert torch.equal(out[f == 0], r[f == 0])


@pytest.mark.parametrize("target", ["x", "residual"])
def test_in_place_and_more_dimensions(target):
    torch, hc = _hc()
    x, r = (torch.randn(3, 5, 41, device="cuda") for _ in range(2))
    want = torch.empty_like(x)
    hc.hc_dropout(x, want, 0.3, 1, 2, residual=r)
    out = x if target == "x" else r
    hc.hc_dropout(x, out, 0.3, 1, 2, residual=r)
    assert torch.equal(out, want)


def test_backward_is_the_same_call():
    torch, hc = _hc()
    rows, cols, p = 37, 45, 0.4
    f = torch.from_numpy(ref.factors(rows, cols, p, 2, 9))
    x = torch.randn(rows, cols, dtype=torch.float64, requires_grad=True)
    dy = torch.randn(rows, cols)
    (x * f).backward(dy.double())
    out = torch.empty(rows, cols, device="cuda")
    hc.hc_dropout(dy.cuda(), out, p, 2, 9)
    assert bool(((out.cpu().double() - x.grad).abs() <= 4 * ref.UNIT * x.grad.abs()).all())


def test_masks_are_uniform_and_differ_by_draw():
    torch, hc = _hc()
    rows, cols = 1024, 1024
    one = torch.ones(rows, cols, device="cuda")
    out = [torch.empty_like(one) for _ in range(3)]
    hc.hc_dropout(one, out[0], 0.25, 1, 0)
    hc.hc_dropout(one, out[1], 0.25, 1, 1)
    hc.hc_dropout(one, out[2], 0.25, 2, 0)
    n = rows * cols
    for o in out:     # 6 standard deviations of a count of n draws
        assert abs(int((o == 0).sum()) - 0.25 * n) < 6 * (n * 0.25 * 0.75) ** 0.5
    for a, b in ((0, 1), (0, 2), (1, 2)):
        same = int(((out[a] == 0) & (out[b] == 0)).sum())
        assert abs(same - n / 16) < 6 * (n / 16 * 15 / 16) ** 0.5


def test_empty_and_offsets_past_32_bits():
    torch, hc = _hc()
    empty = torch.empty(0, 5, device="cuda")
    hc.hc_dropout(empty, empty.clone(), 0.5, 1)
    rows, cols = 2**20 + 3, 4100                    # 4.3e9 elements
    x = torch.ones(rows, cols, device="cuda", dtype=torch.bfloat16)
    hc.hc_dropout(x, x, 0.5, 77, 5)
    for r0 in (0, 1047552, rows - 5):
        got = x[r0:r0 + 5].float().cpu().numpy()
        groups = -(-cols // 8)
        c, r = np.meshgrid(np.arange(groups), np.arange(r0, r0 + 5))
        w = ref.philox([c, r, np.full_like(c, 5), np.zeros_like(c)], (77, 0))
        bits = np.stack([(w[e // 2] >> np.uint64(16 * (e % 2))) & np.uint64(0xFFFF) for e in range(8)], 2)
        want = np.where(bits.reshape(5, groups * 8)[:, :cols] >= 32768, 2.0, 0.0)
        assert np.array_equal(got, want)


def test_counter_moves_the_draw_and_graph_replays_draw_anew():
    torch, hc = _hc()
    x = torch.randn(50, 70, device="cuda")
    counter = torch.zeros(1, device="cuda", dtype=torch.int64)
    out, want = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        hc.hc_dropout(x, out, 0.3, 8, 100, counter=counter)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            hc.hc_dropout(x, out, 0.3, 8, 100, counter=counter)
            counter.add_(1)
    torch.cuda.synchronize()
    counter.zero_()
    seen = []
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        hc.hc_dropout(x, want, 0.3, 8, 100 + i)
        assert torch.equal(out, want)
        seen.append(out.clone())
    assert not torch.equal(seen[0], seen[1])


def test_refusals():
    torch, hc = _hc()
    x = torch.randn(4, 6, device="cuda")
    out = torch.empty_like(x)
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(hc.HCError):
            hc.hc_dropout(x, out, p, 1)
    for bad in (x.cpu(), x[:3], x[:, :5], x.bfloat16(), x.t().contiguous().t()):
        with pytest.raises(ValueError):
            hc.hc_dropout(x, bad, 0.5, 1)
    with pytest.raises(ValueError):
        hc.hc_dropout(x, out, 0.5, 1, counter=torch.zeros(1, device="cuda", dtype=torch.int32))
    wide = torch.empty(4, 12, device="cuda")
    with pytest.raises(hc.HCError):               # in place at another stride
        hc.hc_dropout(wide[:, :6], wide.view(-1)[:24].view(4, 6), 0.5, 1)
