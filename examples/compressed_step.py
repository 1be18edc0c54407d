"""Data-parallel training steps with compressed gradients, end to end on one GPU.

A bag-of-words classifier: token ids are looked up in a scaled embedding table
(hc_embed), the mean of a sequence's rows goes through one weight matrix, and a
cross entropy is taken.  Every simulated worker has its own batch.  Its gradient
is one flat int32 vector in fixed point, the table's part summed by token id
(hc_embed_grad) and the matrix's part behind it.  Workers encode their vectors
(hc_encode), the sketches are summed and the indexes OR-ed (hc_aggregate), and
the exact sum is recovered (hc_decode).  The recovered sum updates the table
directly, and the matrix through its momentum made orthogonal
(hc_orthogonalise), as the Muon optimiser does.

    python examples/compressed_step.py --steps 20
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2402_07529_amd as hc  # noqa: E402

VOCAB, DIM, CLASSES, WORDS, BATCH = 20000, 64, 96, 24, 256
SCALE = DIM**0.5


def batch(gen, meaning):
    """Sequences of words of one class each, an eighth of the places padding (-1)."""
    label = torch.randint(0, CLASSES, (BATCH,), device="cuda", generator=gen)
    pick = torch.randint(0, meaning.shape[1], (BATCH, WORDS), device="cuda", generator=gen)
    ids = meaning[label].gather(1, pick)
    pad = torch.rand(BATCH, WORDS, device="cuda", generator=gen) < 0.125
    return torch.where(pad, -1, ids).to(torch.int32), label


def main(steps=20, workers=4, seed=0, table_lr=20.0, matrix_lr=0.1, momentum=0.9):
    """Runs the steps; returns the mean loss of each."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    meaning = torch.randint(0, VOCAB, (CLASSES, 40), device="cuda", generator=gen)
    table, weight = randn(VOCAB, DIM) * 0.02, randn(CLASSES, DIM) * 0.1
    moment = torch.zeros_like(weight)

    n_table, n = VOCAB * DIM, VOCAB * DIM + CLASSES * DIM
    most = min(n, workers * BATCH * WORDS * DIM + CLASSES * DIM)  # nonzeros of the sum
    p = hc.hc_geometry(n, most, 1.3, 1024, 7, "i32")
    plan = hc.make_plan(p)
    flat = torch.empty((workers, n), device="cuda", dtype=torch.int32)
    y = torch.empty((workers, p.cells), device="cuda", dtype=torch.int32)
    b = torch.empty((workers, p.words), device="cuda", dtype=torch.int32)
    y_sum, b_sum = torch.empty_like(y[0]), torch.empty_like(b[0])
    total = torch.empty(n, device="cuda", dtype=torch.int32)
    info, ws = hc.alloc_info(), hc.alloc_workspace(p, most)
    rows = torch.empty((BATCH, WORDS, DIM), device="cuda")
    grad_ws = hc.alloc_embed_workspace(VOCAB, DIM, BATCH * WORDS)
    ortho_ws, update = hc.alloc_orthogonalise_workspace(weight), torch.empty_like(weight)

    losses = []
    for _ in range(steps):
        loss = 0.0
        for w in range(workers):
            ids, label = batch(gen, meaning)
            hc.hc_embed(table, ids, rows, scale=SCALE)
            x = rows.detach().requires_grad_()
            m = weight.detach().requires_grad_()
            out = torch.nn.functional.cross_entropy(x.mean(1) @ m.t(), label)
            out.backward()
            loss += out.detach() / workers
            hc.hc_embed_grad(x.grad, ids, flat[w, :n_table].view(VOCAB, DIM), grad_ws, scale=SCALE)
            flat[w, n_table:] = torch.round(m.grad * hc.FIXED_POINT).to(torch.int32).view(-1)
            hc.hc_encode(p, flat[w], y[w], b[w])
        hc.hc_aggregate(p, y, b, workers, y_sum, b_sum)
        hc.hc_decode(p, y_sum, b_sum, info, ws, x_out=total, max_support=most, plan=plan)
        assert hc.read_info(info).success, "the sketch was too small for the sum"
        grad = total.float() / (hc.FIXED_POINT * workers)
        table.sub_(grad[:n_table].view(VOCAB, DIM), alpha=table_lr)
        moment.mul_(momentum).add_(grad[n_table:].view_as(moment))
        hc.hc_orthogonalise(moment, update, ortho_ws, scale=(CLASSES / DIM) ** 0.5)
        weight.sub_(update, alpha=matrix_lr)
        losses.append(float(loss))
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--workers", type=int, default=4)
    a = ap.parse_args()
    for step, value in enumerate(main(a.steps, a.workers)):
        print(f"step {step}: loss {value:.4f}", flush=True)
