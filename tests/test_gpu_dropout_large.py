"""Dropout of many elements: four groups of eight a lane, through the caches and past them, in every type,
with rows that end inside a lane's step.  Tolerance as in test_gpu_dropout."""
import functools

import pytest

import layer_reference as ref
from test_gpu_dropout import _check, _hc, _strided

pytestmark = pytest.mark.gpu

SEED, DRAW, P = 0x9876543210ABCDEF, (5 << 34) + 77, 0.3


@functools.lru_cache(maxsize=1)
def _factors(rows, cols):
    import torch
    return torch.from_numpy(ref.factors(rows, cols, P, SEED, DRAW))


# more than 2^18 groups of eight; the last two are more than 32 MB in every type
@pytest.mark.parametrize("rows,cols", [(3001, 771), (270001, 5), (3, 800003), (16384, 1100), (4111, 4109)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("gap,offset", [(0, 0), (5, 3)])
@pytest.mark.parametrize("with_residual", [False, True])
def test_many_elements(rows, cols, dtype, gap, offset, with_residual):
    torch, hc = _hc()
    gen, dt = torch.Generator().manual_seed(rows), getattr(torch, dtype)
    f = _factors(rows, cols)
    _, x = _strided(torch, rows, cols, gap, offset, dt, gen)
    residual = _strided(torch, rows, cols, gap + 3, offset, dt, gen)[1] if with_residual else None
    flat, out = _strided(torch, rows, cols, gap, offset, dt)
    before = flat.clone()
    hc.hc_dropout(x, out, P, SEED, DRAW, residual=residual)
    _check(torch, out.cpu(), x.cpu().double(), None if residual is None else residual.cpu().double(), f, dtype)
    # in place
    target = x if residual is None else residual
    hc.hc_dropout(x, target, P, SEED, DRAW, residual=residual)
    assert torch.equal(target, out)
    out.copy_(before.as_strided(out.shape, out.stride(), offset))
    assert torch.equal(flat, before), "wrote outside its rows"
