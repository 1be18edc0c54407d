"""hc_linear and hc_linear_grad refuse outputs that are another's, before anything is enqueued: two
workgroups would write, or read and write, the same place."""
import ctypes

import pytest

from test_layer_abi import A, B, C, E, F, _backward, _forward, _linear


@pytest.mark.parametrize("kw", [dict(y=C), dict(z=C), dict(z=E)])
def test_forward_outputs_are_apart(kw):
    import paper_2402_07529_amd as hc
    L = hc.lib()
    assert _forward(L, ctypes.byref(_linear(hc)), **kw) == hc.HC_EINVAL
    assert b"overlap" in L.hc_last_error()


@pytest.mark.parametrize("kw", [dict(dw=E), dict(db=E), dict(db=F), dict(dx=F), dict(dw=E, db=None),
                                dict(dx=None, db=F)])
@pytest.mark.parametrize("g", [0, 1, 2])
def test_gradients_are_apart(kw, g):
    import paper_2402_07529_amd as hc
    L = hc.lib()
    assert _backward(L, ctypes.byref(_linear(hc)), g=g, **kw) == hc.HC_EINVAL
    assert b"overlap" in L.hc_last_error()


def test_no_rows_have_no_input_gradient_to_overlap():
    """Without rows dx is not written: an empty dx may have any address."""
    import paper_2402_07529_amd as hc
    L = hc.lib()
    assert _backward(L, ctypes.byref(_linear(hc, m=0)), dx=F, size=0) == hc.HC_EWORKSPACE
    assert _backward(L, ctypes.byref(_linear(hc, m=0)), db=F) == hc.HC_EINVAL
