"""hc_dropout, hc_linear and hc_linear_grad on the host: invalid arguments are refused, with a
message, before anything is enqueued; and the tests' generator gives its published vectors."""
import ctypes

import pytest

import layer_reference as ref

V = ctypes.c_void_p
A, B, C, D, E, F, G, W = (V(4096 * i) for i in range(1, 9))


def test_reference_generator_gives_the_published_vectors():
    low = 0xFFFFFFFF
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((low,) * 4, (low, low), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
             (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(v) for v in ref.philox(counter, key)) == want


def _dropout(hc, **kw):
    d = dict(rows=10, cols=16, x_ld=16, residual_ld=16, out_ld=16, seed=1, draw=2, p=0.5, reserved=0)
    d.update(kw)
    return hc.hc_dropout_params(**d)


@pytest.mark.parametrize("kw", [
    dict(rows=2**31), dict(cols=0), dict(cols=2**31, x_ld=2**31, residual_ld=2**31, out_ld=2**31),
    dict(rows=2**30, cols=2**9, x_ld=2**9, residual_ld=2**9, out_ld=2**9), dict(x_ld=15), dict(out_ld=15),
    dict(residual_ld=15), dict(x_ld=2**31 + 1), dict(p=-1e-9), dict(p=1.0001), dict(p=float("nan")),
    dict(reserved=1)])
def test_dropout_params_refused(kw):
    import paper_2402_07529_amd as hc
    p = _dropout(hc, **kw)
    assert hc.lib().hc_dropout(ctypes.byref(p), 1, A, B, C, None, None) == hc.HC_EINVAL
    assert hc.lib().hc_last_error()


def test_dropout_buffers_refused():
    import paper_2402_07529_amd as hc
    L, p = hc.lib(), _dropout(hc)
    r = ctypes.byref(p)
    assert L.hc_dropout(None, 1, A, B, C, None, None) == hc.HC_EINVAL
    for t in (hc.HC_T_I32, 4, -1):
        assert L.hc_dropout(r, t, A, B, C, None, None) == hc.HC_EINVAL
    for x, res, out, counter in ((None, B, C, None), (A, B, None, None), (V(4098), B, C, None),
                                 (A, V(4098), C, None), (A, B, V(4098), None), (A, B, C, V(4100))):
        assert L.hc_dropout(r, 1, x, res, out, counter, None) == hc.HC_EINVAL
    for same in (dict(x_ld=17), dict(residual_ld=17)):   # in place at another stride
        q = _dropout(hc, **same)
        out = A if "x_ld" in same else B
        assert L.hc_dropout(ctypes.byref(q), 1, A, B, out, None, None) == hc.HC_EINVAL
    none = _dropout(hc, rows=0)
    assert L.hc_dropout(ctypes.byref(none), 1, None, None, None, None, None) == hc.HC_OK


def _linear(hc, **kw):
    d = dict(m=20, n=12, k=16, x_ld=16, w_ld=16, y_ld=12, z_ld=12, residual_ld=12, dx_ld=16, dw_ld=16, seed=0,
             draw=0, p=0.1, act=2, fixed=1.0, reserved=0)
    d.update(kw)
    return hc.hc_linear_params(**d)


def _forward(L, r, t=1, x=A, w=B, bias=C, residual=D, y=E, z=F, counter=None, ws=W, size=2**40):
    return L.hc_linear(r, t, x, w, bias, residual, y, z, counter, ws, size, None)


def _backward(L, r, t=1, dy=A, x=B, w=C, z=D, dx=E, g=1, dw=F, db=G, acc=0, counter=None, ws=W, size=2**40):
    return L.hc_linear_grad(r, t, dy, x, w, z, dx, g, dw, db, acc, counter, ws, size, None)


@pytest.mark.parametrize("kw", [
    dict(m=2**31), dict(n=0), dict(k=0), dict(n=2**24 + 1, y_ld=2**25, z_ld=2**25, residual_ld=2**25),
    dict(k=2**24 + 1, x_ld=2**25, w_ld=2**25, dx_ld=2**25, dw_ld=2**25),
    dict(m=2**30, n=2**9, y_ld=2**9, z_ld=2**9, residual_ld=2**9), dict(x_ld=15), dict(w_ld=15), dict(y_ld=11),
    dict(x_ld=2**31 + 1), dict(act=6), dict(p=2.0), dict(p=float("nan")), dict(reserved=3)])
def test_linear_params_refused(kw):
    import paper_2402_07529_amd as hc
    L, size = hc.lib(), ctypes.c_size_t()
    r = ctypes.byref(_linear(hc, **kw))
    assert L.hc_linear_bytes(r, 1, ctypes.byref(size)) == hc.HC_EINVAL and L.hc_last_error()
    assert L.hc_linear_grad_bytes(r, 1, ctypes.byref(size)) == hc.HC_EINVAL
    assert _forward(L, r) == hc.HC_EINVAL
    assert _backward(L, r) == hc.HC_EINVAL


def test_linear_buffers_refused():
    import paper_2402_07529_amd as hc
    L, size = hc.lib(), ctypes.c_size_t()
    r = ctypes.byref(_linear(hc))
    assert L.hc_linear_bytes(r, 1, None) == hc.HC_EINVAL
    assert L.hc_linear_bytes(r, 0, ctypes.byref(size)) == hc.HC_EINVAL
    assert L.hc_linear_bytes(r, 1, ctypes.byref(size)) == hc.HC_OK and size.value > 0
    assert _forward(L, r, size=size.value - 1) == hc.HC_EWORKSPACE
    for kw in (dict(t=0), dict(t=4), dict(x=None), dict(w=None), dict(y=None), dict(ws=None), dict(ws=V(128)),
               dict(x=V(4098)), dict(w=V(4098)), dict(bias=V(4098)), dict(residual=V(4098)), dict(y=V(4098)),
               dict(z=V(4098)), dict(counter=V(4100)), dict(y=A), dict(y=B), dict(z=E), dict(z=A), dict(z=D)):
        assert _forward(L, r, **kw) == hc.HC_EINVAL, kw
    for kw in (dict(z_ld=11), dict(residual_ld=11), dict(residual_ld=13)):
        q = ctypes.byref(_linear(hc, **kw))
        assert _forward(L, q, y=D if kw == dict(residual_ld=13) else E) == hc.HC_EINVAL, kw
    assert _forward(L, ctypes.byref(_linear(hc, m=0)), x=None, w=None, y=None, ws=None) == hc.HC_OK


def test_gradient_buffers_refused():
    import paper_2402_07529_amd as hc
    L, size = hc.lib(), ctypes.c_size_t()
    r = ctypes.byref(_linear(hc))
    assert L.hc_linear_grad_bytes(r, 1, None) == hc.HC_EINVAL
    assert L.hc_linear_grad_bytes(r, 1, ctypes.byref(size)) == hc.HC_OK and size.value > 0
    assert _backward(L, r, size=size.value - 1) == hc.HC_EWORKSPACE
    for kw in (dict(t=0), dict(g=4), dict(g=-1), dict(dy=None), dict(x=None), dict(w=None), dict(z=None),
               dict(ws=None), dict(ws=V(128)), dict(dy=V(4098)), dict(x=V(4098)), dict(w=V(4098)), dict(z=V(4098)),
               dict(dx=V(4098)), dict(dw=V(4098)), dict(db=V(4098)), dict(counter=V(4100)), dict(dx=A), dict(dx=B),
               dict(dw=C), dict(db=D)):
        assert _backward(L, r, **kw) == hc.HC_EINVAL, kw
    for kw in (dict(z_ld=11), dict(dx_ld=15), dict(dw_ld=15)):
        assert _backward(L, ctypes.byref(_linear(hc, **kw))) == hc.HC_EINVAL, kw
    for fixed in (0.0, -1.0, float("inf"), float("nan")):
        assert _backward(L, ctypes.byref(_linear(hc, fixed=fixed)), g=0) == hc.HC_EINVAL


@pytest.mark.parametrize("n,k", [(12, 16), (768, 768), (33278, 1500), (64, 128), (4096, 25088), (7, 3)])
@pytest.mark.parametrize("t", [1, 2, 3])
def test_a_workspace_does_for_fewer_rows(n, k, t):
    import paper_2402_07529_amd as hc
    L, size = hc.lib(), ctypes.c_size_t()
    for call in (L.hc_linear_bytes, L.hc_linear_grad_bytes):
        last = 0
        for m in sorted({1, 2, 15, 16, 17, 33, 63, 64, 65, 127, 129, 255, 256, 257, 700, 1000, 2047, 4096, 5000, 10000,
                         32768, 65536, 100000}):
            p = _linear(hc, m=m, n=n, k=k, x_ld=k, w_ld=k, y_ld=n, z_ld=n, residual_ld=n, dx_ld=k, dw_ld=k)
            assert call(ctypes.byref(p), t, ctypes.byref(size)) == hc.HC_OK
            assert size.value >= last, m
            last = size.value


def test_binding_refuses_host_tensors_and_unknown_names():
    torch = pytest.importorskip("torch")
    import paper_2402_07529_amd as hc
    x, w, y, ws = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(4, 6), torch.zeros(512, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device tensor"):
        hc.hc_dropout(x, x.clone(), 0.5, 1)
    with pytest.raises(ValueError, match="device tensor"):
        hc.hc_linear(x, w, y, ws)
    with pytest.raises(ValueError, match="device tensor"):
        hc.hc_linear_grad(y, ws, x=x, dw=w)
    with pytest.raises(ValueError, match="device tensor"):
        hc.alloc_linear_workspace(x, w)
    assert set(hc.ACTIVATIONS) == {"none", "relu", "gelu", "silu", "tanh", "sigmoid"}
