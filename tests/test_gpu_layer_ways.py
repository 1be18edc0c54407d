"""A gradient of the linear layer is the same, bit for bit, whichever others are wanted beside it: by each
way that a product goes, and with operands of other strides and addresses."""
import pytest

from test_gpu_linear import TYPES, Layer, _hc

pytestmark = pytest.mark.gpu


def _shifted(torch, t, gap, offset):
    """t's values in rows `gap` elements further apart, `offset` elements behind a 256-byte address."""
    rows, cols = t.shape
    flat = torch.full((offset + rows * (cols + gap) + 8,), float("nan"), device="cuda", dtype=t.dtype)
    return flat.as_strided((rows, cols), (cols + gap, 1), offset).copy_(t)


# small products for dx beside tiles or direct ones for dw, both in tiles, both small, copied operands
ALONE = [(16, 768, 768), (64, 768, 768), (1, 4096, 4096), (512, 768, 768), (600, 96, 64), (1100, 1000, 1300),
         (1200, 1024, 1024), (33, 70, 1001)]


@pytest.mark.parametrize("m,n,k", ALONE)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_a_gradient_is_the_same_alone(m, n, k, dtype, act):
    torch, hc = _hc()
    L = Layer(torch, m, n, k, dtype)
    kw = dict(act=act, p=0.1 if act == "gelu" else 0.0, seed=7, draw=k)
    if act == "gelu":
        kw["z"] = L.z
    # (gap, offset) of x, w and dy
    for x_at, w_at, dy_at in (((0, 0), (0, 0), (0, 0)), ((0, 1), (0, 0), (0, 0)), ((0, 0), (0, 1), (0, 1)),
                              ((3, 0), (0, 1), (0, 0)), ((0, 1), (5, 0), (2, 0))):
        x, w, dy = _shifted(torch, L.x, *x_at), _shifted(torch, L.w, *w_at), _shifted(torch, L.dy, *dy_at)
        ws = hc.alloc_linear_grad_workspace(x, w)
        for out in ("float32", dtype):
            wide = getattr(torch, out)

            def outs():
                return (torch.full_like(L.x, 9), torch.full((n, k), 9.0, device="cuda", dtype=wide),
                        torch.full((n,), 9.0, device="cuda", dtype=wide))

            dx, dw, db = outs()
            hc.hc_linear_grad(dy, ws, x=x, w=w, dx=dx, dw=dw, db=db, **kw)
            ax, aw, ab = outs()
            bx, bw, bb = outs()
            hc.hc_linear_grad(dy, ws, w=w, dx=ax, **kw)
            hc.hc_linear_grad(dy, ws, x=x, dw=aw, **kw)
            hc.hc_linear_grad(dy, ws, db=ab, **kw)
            hc.hc_linear_grad(dy, ws, x=x, w=w, dx=bx, db=bb, **kw)
            hc.hc_linear_grad(dy, ws, x=x, dw=bw, **kw)
            where = (x_at, w_at, dy_at, out)
            assert torch.equal(dx, ax) and torch.equal(dx, bx), ("dx", where)
            assert torch.equal(dw, aw) and torch.equal(dw, bw), ("dw", where)
            assert torch.equal(db, ab) and torch.equal(db, bb), ("db", where)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_small_and_large_products_of_a_call_captured_and_replayed(dtype, act):
    """dx and db small beside a dw in tiles, in a graph, against the eager call."""
    torch, hc = _hc()
    L = Layer(torch, 16, 768, 768, dtype)
    ws = hc.alloc_linear_grad_workspace(L.x, L.w)
    kw = dict(x=L.x, w=L.w, z=L.z if act != "none" else None, act=act, p=0.2 if act == "gelu" else 0.0, seed=3)

    def outs():
        return dict(dx=torch.empty_like(L.x), dw=torch.empty(768, 768, device="cuda"),
                    db=torch.empty(768, device="cuda"))

    got, want, side, graph = outs(), outs(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    hc.hc_linear_grad(L.dy, ws, **kw, **got)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        hc.hc_linear_grad(L.dy, ws, **kw, **got)
    for _ in range(3):
        L.dy.mul_(0.5)         # eager work between the replays
        for t in got.values():
            t.fill_(float("nan"))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        hc.hc_linear_grad(L.dy, ws, **kw, **want)
        assert all(torch.equal(got[name], want[name]) for name in got)
        torch.cuda.synchronize()
