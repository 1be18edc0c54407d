"""A worker's gradient in examples/compressed_step.py, through lookup, dropout and layer, against
autograd in 64 bits.

Tolerance: the layer's and the table's sums are rounded to whole units of 2^-20 (a unit for each of the
table's terms), and fp32 leaves (terms + 8) 2^-24 of the sums of magnitudes, loosely bounded by the
largest gradient."""
import importlib.util
import os

import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_worker_gradient():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location(
        "compressed_step", os.path.join(ROOT, "examples", "compressed_step.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    meaning = torch.randint(0, ex.VOCAB, (ex.CLASSES, 40), device="cuda", generator=gen)
    table = torch.randn(ex.VOCAB, ex.DIM, device="cuda", generator=gen) * 0.02
    weight = torch.randn(ex.CLASSES, ex.DIM, device="cuda", generator=gen) * 0.1
    ids, label = ex.batch(gen, meaning)
    n_table = ex.VOCAB * ex.DIM
    flat = torch.empty(n_table + ex.CLASSES * ex.DIM, device="cuda", dtype=torch.int32)
    loss = ex.Worker(11).gradient(table, weight, ids, label, 5, flat)

    t, w = (v.cpu().double().requires_grad_() for v in (table, weight))
    i, lab = ids.cpu().long(), label.cpu()
    rows = torch.where((i >= 0)[..., None], t[i.clamp(min=0)] * ex.SCALE, 0.0)
    f = torch.from_numpy(ref.factors(ex.BATCH, ex.DIM, ex.DROP, 11, 5))
    want = torch.nn.functional.cross_entropy((rows.mean(1) * f) @ w.t(), lab)
    want.backward()
    assert abs(float(loss) - float(want.detach())) < 1e-5
    unit = 2.0**-20
    got = flat.cpu().double() * unit
    count = torch.bincount(i[i >= 0].reshape(-1), minlength=ex.VOCAB).double()[:, None]
    most = float(t.grad.abs().max())
    off = (got[:n_table].view_as(t.grad) - t.grad).abs()
    assert bool((off <= count * (0.5 * unit + 200 * ref.UNIT * most)).all())
    off = (got[n_table:].view_as(w.grad) - w.grad).abs()
    assert bool((off <= 0.5 * unit + (ex.BATCH + 200) * ref.UNIT * float(w.grad.abs().max())).all())
