"""include/hc_train.h on the host: every declared entry point is exported, and
invalid arguments are refused, with a message, before anything is enqueued."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
V = ctypes.c_void_p


def test_library_exports_every_declared_symbol():
    import paper_2402_07529_amd as hc
    with open(os.path.join(ROOT, "include", "hc_train.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = set(re.findall(r"\b(hc_[a-z_0-9]+)\s*\(", text))
    assert names == set(hc.TRAIN_EXPORTS)
    lib = ctypes.CDLL(hc.LIB_PATH)
    for name in names:
        assert hasattr(lib, name), name


def _embed(hc, **kw):
    d = dict(vocab=100, count=10, dim=16, table_ld=16, x_ld=16, padding=-1, id_bits=32, reserved=0,
             scale=1.0, fixed=2.0**20)
    d.update(kw)
    return hc.hc_embed_params(**d)


BAD_EMBED = [dict(vocab=0), dict(vocab=2**31), dict(count=2**31), dict(dim=0), dict(dim=2**22 + 1),
             dict(table_ld=15), dict(x_ld=15), dict(x_ld=2**31 + 1), dict(id_bits=16),
             dict(reserved=1), dict(scale=float("inf")), dict(scale=float("nan"))]


@pytest.mark.parametrize("kw", BAD_EMBED)
def test_embed_params_refused(kw):
    import paper_2402_07529_amd as hc
    L, p = hc.lib(), _embed(hc, **kw)
    size = ctypes.c_size_t()
    r = ctypes.byref(p)
    assert L.hc_embed(r, hc.HC_T_F32, V(256), V(256), V(256), None) == hc.HC_EINVAL
    assert L.hc_last_error()
    assert L.hc_embed_grad_bytes(r, ctypes.byref(size)) == hc.HC_EINVAL
    assert L.hc_embed_grad(r, hc.HC_T_F32, V(256), V(256), hc.HC_T_F32, V(256), 0, V(256),
                           2**40, None) == hc.HC_EINVAL
    assert L.hc_embed_grad_rows(r, hc.HC_T_F32, V(256), V(256), hc.HC_T_F32, V(256), V(256), 10,
                                V(256), V(256), 2**40, None) == hc.HC_EINVAL


def test_embed_buffers_refused():
    import paper_2402_07529_amd as hc
    L, p = hc.lib(), _embed(hc)
    r = ctypes.byref(p)
    assert L.hc_embed(None, 1, V(256), V(256), V(256), None) == hc.HC_EINVAL
    for bad in ((None, V(256), V(256)), (V(256), None, V(256)), (V(256), V(256), None),
                (V(258), V(256), V(256)), (V(256), V(258), V(256)), (V(256), V(256), V(257))):
        assert L.hc_embed(r, hc.HC_T_F32, *bad, None) == hc.HC_EINVAL
    for t in (hc.HC_T_I32, 4, -1):
        assert L.hc_embed(r, t, V(256), V(256), V(256), None) == hc.HC_EINVAL
    size = ctypes.c_size_t()
    assert L.hc_embed_grad_bytes(r, ctypes.byref(size)) == hc.HC_OK and size.value > 0
    assert L.hc_embed_grad_bytes(r, None) == hc.HC_EINVAL

    def grad(x_type=1, dout=V(256), ids=V(256), g_type=1, dst=V(256), ws=V(256), n=2**40):
        return L.hc_embed_grad(r, x_type, dout, ids, g_type, dst, 0, ws, n, None)

    for kw in (dict(x_type=0), dict(x_type=4), dict(g_type=4), dict(dout=None), dict(ids=None),
               dict(dst=None), dict(ws=None), dict(ws=V(128)), dict(dout=V(258)), dict(ids=V(258)),
               dict(dst=V(258))):
        assert grad(**kw) == hc.HC_EINVAL, kw
    assert grad(n=size.value - 1) == hc.HC_EWORKSPACE
    for fixed in (0.0, -1.0, float("inf"), float("nan")):
        q = _embed(hc, fixed=fixed)
        assert L.hc_embed_grad(ctypes.byref(q), 1, V(256), V(256), hc.HC_T_I32, V(256), 0, V(256),
                               2**40, None) == hc.HC_EINVAL
    for rows, touched in ((None, V(256)), (V(256), None), (V(258), V(256)), (V(256), V(257))):
        assert L.hc_embed_grad_rows(r, 1, V(256), V(256), 1, rows, V(256), 10, touched, V(256), 2**40,
                                    None) == hc.HC_EINVAL
    # a gradient call takes at most 2^30 ids
    assert L.hc_embed_grad_bytes(ctypes.byref(_embed(hc, count=2**30 + 1)),
                                 ctypes.byref(size)) == hc.HC_EINVAL
    # no ids: nothing to look up, nothing enqueued
    assert L.hc_embed(ctypes.byref(_embed(hc, count=0)), 1, V(256), None, None, None) == hc.HC_OK


def _ortho(hc, **kw):
    d = dict(m=64, n=96, batch=1, x_ld=96, x_stride=0, out_ld=96, out_stride=0, type=hc.HC_T_F32,
             steps=5, coeffs=None, eps=1e-7, scale=1.0)
    d.update(kw)
    if d["coeffs"] is not None:
        d["coeffs"] = (ctypes.c_float * len(d["coeffs"]))(*d["coeffs"])
    return hc.hc_orthogonalise_params(**d)


@pytest.mark.parametrize("kw", [
    dict(m=0), dict(n=0), dict(m=65537), dict(n=65537, x_ld=65537, out_ld=65537),
    dict(batch=65536, out_stride=64 * 96), dict(x_ld=95), dict(out_ld=95), dict(x_ld=2**40 + 1),
    dict(batch=2, out_stride=64 * 96 - 1), dict(type=0), dict(type=3), dict(steps=33),
    dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(scale=float("inf")),
    dict(steps=1, coeffs=[1.0, float("nan"), 0.0])])
def test_orthogonalise_params_refused(kw):
    import paper_2402_07529_amd as hc
    L, p = hc.lib(), _ortho(hc, **kw)
    size = ctypes.c_size_t()
    assert L.hc_orthogonalise_bytes(ctypes.byref(p), ctypes.byref(size)) == hc.HC_EINVAL
    assert L.hc_last_error()
    assert L.hc_orthogonalise(ctypes.byref(p), V(256), V(256), V(256), 2**50, None) == hc.HC_EINVAL


@pytest.mark.parametrize("coeffs", [(2000.0, 0.0, 0.0), (0.0, 0.0, 0.0), (1e-4, 0.0, 0.0),
                                    (1.0, 0.0, 2000.0), (1.0, 5000.0, -5000.0)])
def test_orthogonalise_coefficients_out_of_range(coeffs):
    import paper_2402_07529_amd as hc
    p = _ortho(hc, steps=1, coeffs=coeffs)
    size = ctypes.c_size_t()
    assert hc.lib().hc_orthogonalise_bytes(ctypes.byref(p), ctypes.byref(size)) == hc.HC_EUNSUPPORTED


def test_orthogonalise_buffers_refused():
    import paper_2402_07529_amd as hc
    L, p = hc.lib(), _ortho(hc)
    r, size = ctypes.byref(p), ctypes.c_size_t()
    assert L.hc_orthogonalise_bytes(r, ctypes.byref(size)) == hc.HC_OK
    assert L.hc_orthogonalise_bytes(None, ctypes.byref(size)) == hc.HC_EINVAL
    assert L.hc_orthogonalise_bytes(r, None) == hc.HC_EINVAL
    n = size.value
    for bad in ((None, V(256), V(256)), (V(256), None, V(256)), (V(256), V(256), None),
                (V(258), V(256), V(256)), (V(256), V(258), V(256)), (V(256), V(256), V(128))):
        assert L.hc_orthogonalise(r, *bad, n, None) == hc.HC_EINVAL
    assert L.hc_orthogonalise(r, V(256), V(256), V(256), n - 1, None) == hc.HC_EWORKSPACE
    assert L.hc_orthogonalise(ctypes.byref(_ortho(hc, batch=0)), None, None, None, 0, None) == hc.HC_OK


def test_binding_refuses_host_tensors_and_shapes():
    import torch
    import paper_2402_07529_amd as hc
    t = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        hc.hc_embed(t, torch.zeros(2, dtype=torch.int32), torch.zeros(2, 8))
    with pytest.raises(ValueError):
        hc.hc_embed_grad(t, torch.zeros(4, dtype=torch.int32), t, torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(ValueError):
        hc.hc_orthogonalise(t, t.clone(), torch.zeros(256, dtype=torch.uint8))


@pytest.mark.parametrize("dim", [1, 4, 5, 16, 64, 100, 768, 1500, 5000])
def test_gradient_workspace_grows_with_the_count(dim):
    """A workspace for up to `count` ids does for any smaller number of them."""
    import paper_2402_07529_amd as hc
    last, count = 0, 0
    while count < 2**22:
        need = hc.hc_embed_grad_bytes(70000, dim, count)
        assert need >= last, (dim, count)
        last = need
        count += max(1, count // 37)
    for edge in (8192, 2**19, 2**20):
        sizes = [hc.hc_embed_grad_bytes(70000, dim, edge + k) for k in range(-3, 4)]
        assert sizes == sorted(sizes)


def test_chunks_fit_their_bound():
    """What a call lays out never needs more than what the bytes call reported for it: counts at
    and around where the split changes."""
    import paper_2402_07529_amd as hc
    for dim in (1, 3, 17, 64, 65, 513, 1500):
        for count in [2**k + d for k in range(3, 21) for d in (-1, 0, 1)]:
            # two partial sums of dim elements a chunk of at most 64 pairs, and the sorted pairs
            assert hc.hc_embed_grad_bytes(1000, dim, count) >= count * 8 + -(-count // 64) * 16 * dim


@pytest.mark.parametrize("m,n", [(64, 96), (200, 300), (768, 768), (5000, 257)])
def test_an_empty_batch_needs_no_workspace(m, n):
    """0 bytes for no matrices, at sides of every plan.  In a process of its own: the size was a
    division by zero for shorter sides above 128."""
    code = ("import ctypes, paper_2402_07529_amd as hc\n"
            "for t in (hc.HC_T_F32, hc.HC_T_BF16):\n"
            f"    p = hc.hc_orthogonalise_params({m}, {n}, 0, {n}, 0, {n}, 0, t, 5, None, 1e-7, 1.0)\n"
            "    size = ctypes.c_size_t(7)\n"
            "    assert hc.lib().hc_orthogonalise_bytes(ctypes.byref(p), ctypes.byref(size)) == hc.HC_OK\n"
            "    assert size.value == 0\n")
    got = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert got.returncode == 0, (got.returncode, got.stderr)


def test_output_matrices_may_interleave_by_rows():
    """Row i of all matrices before any row i + 1, as a [m, batch, n] tensor holds them, does not overlap."""
    import paper_2402_07529_amd as hc
    size = ctypes.c_size_t()
    for m, n, batch, ld, stride, ok in ((64, 96, 3, 288, 96, True), (64, 96, 3, 287, 96, False),
                                        (64, 96, 3, 288, 95, False), (64, 96, 3, 300, 102, True),
                                        (64, 96, 3, 300, 103, False), (1, 96, 3, 96, 96, True),
                                        (1, 96, 3, 96, 95, False), (64, 96, 65535, 2**40, 2**24, True)):
        p = _ortho(hc, m=m, n=n, batch=batch, x_ld=n, out_ld=ld, out_stride=stride)
        want = hc.HC_OK if ok else hc.HC_EINVAL
        assert hc.lib().hc_orthogonalise_bytes(ctypes.byref(p), ctypes.byref(size)) == want, (ld, stride)


def _gradient_needs(dim, count):
    """Bytes that a gradient of `count` ids touches, by how it splits them: sorted pairs, the sort's
    own list (and, past 32,768 ids, 512 counts a workgroup), and for each chunk of pairs a head count, a
    shared run and two partial sums of 64-bit elements."""
    def group(vectors):
        if vectors > 64 and 16 < vectors % 64 <= 32:
            return 32
        return 1 << min(6, (vectors - 1).bit_length())

    def up(v, a):
        return -(-v // a) * a

    chunk, row = 64, -(-dim // 8)
    while chunk > 8 and chunk * 256 // group(row) > 2048:
        chunk //= 2
    lanes = up(-(-dim // 4), group(-(-dim // 4)))
    while chunk > 4 and count // chunk * lanes // 64 < 4096:
        chunk //= 2
    chunks = -(-count // chunk)
    need = up(count * 8, 256) + up(512 * 4, 256) + 256
    if 6144 < count <= 32768:
        need += 2 * up(count * 4, 256)
    elif count > 32768:
        threads = 512 if count >= 2**19 else 256
        need += up(count * 8, 256) + up(-(-count // (threads * 8)) * 512 * 4, 256)
    return need + up(chunks * 4, 256) + up(chunks * 8, 256) + up(chunks * 2 * up(dim, 8) * 8, 256)


@pytest.mark.parametrize("dim", [1, 3, 17, 64, 65, 513, 640, 768, 1500, 2100, 5000])
def test_workspace_holds_what_a_gradient_touches(dim):
    """What is reported for a number of ids is enough for it and for every smaller number, around
    every place where chunks, sorting workgroups or the sort itself change."""
    import paper_2402_07529_amd as hc
    edges = {1, 2, 3, 5, 6144, 8192, 32768, 2**19, 2**20}
    edges |= {2**k for k in range(3, 22)} | {3 * 2**k for k in range(2, 20)}
    lanes = -(-dim // 4)
    for chunk in (4, 8, 16, 32, 64):        # a chunk is halved until it leaves 4096 waves
        for per_row in (lanes, lanes + 31, lanes + 63):
            edges.add(chunk * 64 * 4096 // per_row)
    counts = sorted({e + d for e in edges for d in (-65, -1, 0, 1, 64) if 0 < e + d <= 2**22})
    most = 0
    for count in counts:
        most = max(most, _gradient_needs(dim, count))
        assert hc.hc_embed_grad_bytes(70000, dim, count) >= most, count
    for edge in (6144, 32768):
        sizes = [hc.hc_embed_grad_bytes(70000, dim, edge + k) for k in range(-3, 4)]
        assert sizes == sorted(sizes)
