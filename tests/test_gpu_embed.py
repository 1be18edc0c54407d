"""Embedding lookup and its gradient against plain formulas in 64 bits.

Tolerances, from the arithmetic: a lookup is one fp32 product rounded once, so
it equals torch's bit for bit.  A row's gradient is a sum of t fp32 products
(2^-24 relative each, t of them and t - 1 sums, in whatever grouping), so an
element is within (t + 2) 2^-24 of the sum of its terms' magnitudes, plus half
a unit of its type where it is rounded to fewer bits.  Fixed point is exact."""
import pytest

pytestmark = pytest.mark.gpu

HALF_UNIT = {"float32": 2.0**-24, "bfloat16": 2.0**-8, "float16": 2.0**-11}


def _hc():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2402_07529_amd as hc
    return torch, hc


def _ids(torch, gen, vocab, count, kind, dtype):
    if kind == "uniform":
        ids = torch.randint(0, vocab, (count,), generator=gen)
    elif kind == "hot":      # nine of ten are one id
        ids = torch.randint(0, vocab, (count,), generator=gen)
        ids[torch.rand(count, generator=gen) < 0.9] = vocab // 2
    elif kind == "one":
        ids = torch.full((count,), vocab - 1)
    elif kind == "invalid":  # none, or every third, inside the table
        ids = torch.randint(0, vocab, (count,), generator=gen)
        ids[::3] = -1
        ids[1::3] = vocab + torch.arange(ids[1::3].numel()) % 5
    else:
        ids = torch.full((count,), -7)
    return ids.to(dtype)


def _strided(torch, rows, cols, gap, offset, dtype):
    """rows x cols with `gap` elements between rows, `offset` elements into its storage."""
    flat = torch.full((offset + rows * (cols + gap) + 8,), 7, device="cuda", dtype=dtype)
    return flat, flat.as_strided((rows, cols), (cols + gap, 1), offset)


LOOKUPS = [(1, 1, 1), (30522, 768, 16), (5, 3, 64), (100, 7, 129), (1000, 33, 300), (33278, 1500, 700),
           (64, 64, 4097), (17, 256, 1000), (9, 1031, 77), (300, 2, 5000), (4, 5000, 3)]


@pytest.mark.parametrize("vocab,dim,count", LOOKUPS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("gap,offset", [(0, 0), (3, 1)])
def test_lookup(vocab, dim, count, dtype, gap, offset):
    torch, hc = _hc()
    gen = torch.Generator().manual_seed(vocab + dim + count)
    dt, scale = getattr(torch, dtype), 3.7
    for kind, it in (("uniform", torch.int32), ("invalid", torch.int64), ("none", torch.int32)):
        ids = _ids(torch, gen, vocab, count, kind, it)
        _, table = _strided(torch, vocab, dim, gap, offset, dt)
        table.copy_(torch.randn(vocab, dim, generator=gen))
        flat, out = _strided(torch, count, dim, gap, offset, dt)
        before = flat.clone()
        hc.hc_embed(table, ids.cuda(), out, scale=scale)
        valid = (ids >= 0) & (ids < vocab)
        want = (table.cpu()[torch.where(valid, ids, 0).long()].float() * scale).to(dt)
        want[~valid] = 0
        assert torch.equal(out.cpu(), want)
        out.copy_(before.as_strided(out.shape, out.stride(), offset))
        assert torch.equal(flat, before), "wrote outside its rows"


def test_lookup_shapes_and_offsets_past_32_bits():
    torch, hc = _hc()
    vocab, dim = 2**23, 520                     # 4.4e9 elements
    table = torch.empty((vocab, dim), device="cuda", dtype=torch.bfloat16)
    at = torch.tensor([0, 1, 8259552, 8259553, vocab - 2, vocab - 1], device="cuda")
    rows = torch.randn(6, dim, device="cuda").bfloat16()
    table[at] = rows
    out = torch.empty((2, 3, dim), device="cuda", dtype=torch.bfloat16)
    hc.hc_embed(table, at.view(2, 3), out)
    assert torch.equal(out.view(6, dim), rows)
    # and the gradient's rows there, added to what they hold
    ws = hc.alloc_embed_workspace(vocab, dim, 6)
    hc.hc_embed_grad(rows, at, table, ws, accumulate=True)
    assert torch.equal(table[at], (rows.float() * 2).bfloat16())


def _reference(torch, dout, ids, vocab, scale, padding):
    """(sum, sum of magnitudes, terms) of every row in 64 bits."""
    ids = ids.long()
    ok = (ids >= 0) & (ids < vocab) & (ids != padding)
    g = dout.double()[ok] * float(torch.tensor(scale))
    zero = torch.zeros((vocab, dout.shape[1]), dtype=torch.float64)
    terms = torch.bincount(ids[ok], minlength=vocab).double()
    return zero.index_add(0, ids[ok], g), zero.index_add(0, ids[ok], g.abs()), terms


def _check(torch, got, want, mag, terms, dtype):
    tol = (terms[:, None] + 2) * 2.0**-24 * mag + HALF_UNIT[dtype] * want.abs()
    if dtype == "float16":
        tol = tol + 2.0**-25   # half of the smallest fp16
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), float((off - tol).max())


GRADS = [  # vocab, dim, count
    (1, 1, 1), (1, 5, 1000), (3, 2, 0), (100, 16, 1), (100, 7, 63), (1000, 33, 64), (50, 64, 65),
    (33278, 100, 700), (257, 300, 2048), (40, 768, 2049), (5000, 64, 8192), (5000, 64, 8193),
    (70000, 8, 30000), (513, 1031, 500), (12, 24, 70001), (2**20 + 3, 4, 20000)]


@pytest.mark.parametrize("vocab,dim,count", GRADS)
@pytest.mark.parametrize("kind", ["uniform", "hot", "one", "invalid", "none"])
@pytest.mark.parametrize("x_type,g_type", [("float32", "float32"), ("bfloat16", "bfloat16"),
                                           ("float16", "float32"), ("bfloat16", "float32"),
                                           ("float32", "float16"), ("float32", "int32"),
                                           ("bfloat16", "int32")])
def test_gradient(vocab, dim, count, kind, x_type, g_type):
    torch, hc = _hc()
    gen = torch.Generator().manual_seed(vocab * 3 + dim + count)
    it = torch.int64 if (vocab + count) % 2 else torch.int32
    ids = _ids(torch, gen, vocab, count, kind, it)
    scale, fixed = 1.3, 2.0**20
    padding = int(ids[0]) if count > 3 and kind == "uniform" else -1
    std = 300.0 if g_type == "int32" and kind == "uniform" else 0.1   # some of it saturates
    dout = (torch.randn(count, dim, generator=gen) * std).to(getattr(torch, x_type))
    gt = getattr(torch, g_type)
    x, d = dout.cuda(), ids.cuda()
    ws = hc.alloc_embed_workspace(vocab, dim, count)
    out = torch.full((vocab, dim), 3, device="cuda", dtype=gt)
    hc.hc_embed_grad(x, d, out, ws, scale=scale, fixed=fixed, padding=padding)
    cap = min(count, vocab)
    rows = torch.full((cap,), -5, device="cuda", dtype=torch.int32)
    values = torch.full((cap, dim), 3, device="cuda", dtype=gt)
    touched = torch.full((1,), -1, device="cuda", dtype=torch.int32)
    hc.hc_embed_grad_rows(x, d, vocab, rows, values, touched, ws, scale=scale, fixed=fixed,
                          padding=padding)

    lid = ids.long()
    ok = (lid >= 0) & (lid < vocab) & (lid != padding)
    distinct = torch.unique(lid[ok])
    n = int(touched)
    assert n == distinct.numel()
    assert torch.equal(rows[:n].cpu().long(), distinct)
    assert bool((rows[n:] == -5).all()) and bool((values[n:] == 3).all())
    got = out.cpu()
    # both forms sum in the same order
    assert torch.equal(values[:n].cpu(), got[distinct])
    untouched = torch.ones(vocab, dtype=torch.bool)
    untouched[distinct] = False
    assert not bool(got[untouched].any())
    if g_type == "int32":
        q = torch.round((dout.float() * torch.tensor(scale)) * fixed).double().clamp(-2.0**31, 2.0**31)
        q = q.to(torch.int64).clamp(-(2**31) + 1, 2**31 - 1)
        want = torch.zeros((vocab, dim), dtype=torch.int64).index_add(0, lid[ok], q[ok])
        assert torch.equal(got.long(), want.clamp(-(2**31) + 1, 2**31 - 1))
    else:
        _check(torch, got, *_reference(torch, dout, ids, vocab, scale, padding), g_type)


@pytest.mark.parametrize("vocab,dim,count", [(5000, 64, 12288), (5000, 64, 12289), (300, 64, 8191), (300, 64, 8193),
                                             (2**24, 4, 12287), (900, 3, 4093), (900, 5, 5),
                                             (2**20, 8, 6144), (77, 8, 6145), (2**24, 3, 7169), (2**24, 2, 32768),
                                             (9000, 2, 32767), (9000, 2, 32769), (2**21, 4, 31745)])
@pytest.mark.parametrize("kind", ["uniform", "hot", "invalid"])
@pytest.mark.parametrize("g_type", ["float32", "int32"])
def test_gradient_either_side_of_a_sort(vocab, dim, count, kind, g_type):
    test_gradient(vocab, dim, count, kind, "float32", g_type)


@pytest.mark.parametrize("vocab,dim,count,gap,offset", [(100, 7, 200, 3, 1), (64, 64, 500, 8, 4),
                                                        (33, 130, 3000, 1, 3)])
@pytest.mark.parametrize("x_type,g_type", [("float32", "float32"), ("bfloat16", "bfloat16"),
                                           ("float16", "int32")])
def test_gradient_strides_and_accumulate(vocab, dim, count, gap, offset, x_type, g_type):
    torch, hc = _hc()
    gen = torch.Generator().manual_seed(count)
    ids = _ids(torch, gen, vocab - 5, count, "invalid", torch.int32)
    ids[ids >= vocab - 5] = -3                       # the last five rows stay untouched
    gt = getattr(torch, g_type)
    _, x = _strided(torch, count, dim, gap, offset, getattr(torch, x_type))
    x.copy_(torch.randn(count, dim, generator=gen))
    flat, out = _strided(torch, vocab, dim, gap, offset, gt)
    outside = flat.clone()
    ws = hc.alloc_embed_workspace(vocab, dim, count)
    hc.hc_embed_grad(x, ids.cuda(), out, ws)
    want, mag, terms = _reference(torch, x.cpu(), ids, vocab, 1.0, -1)
    if g_type == "int32":
        q = torch.round(x.cpu().float() * 2.0**20).to(torch.int64)
        ok = ids >= 0
        exact = torch.zeros((vocab, dim), dtype=torch.int64).index_add(0, ids[ok].long(), q[ok])
        assert torch.equal(out.cpu().long(), exact)
    else:
        _check(torch, out.cpu(), want, mag, terms, g_type)
    first = out.clone()
    hc.hc_embed_grad(x, ids.cuda(), out, ws, accumulate=True)
    if g_type == "int32":
        assert torch.equal(out.cpu().long(), 2 * exact)
    else:
        base = first.cpu().double()
        # one more fp32 sum, and the rounding of the result
        _check(torch, out.cpu(), want + base, mag + base.abs(), terms + 1, g_type)
    assert torch.equal(out[-5:], first[-5:])
    out.copy_(outside.as_strided(out.shape, out.stride(), offset))
    assert torch.equal(flat, outside), "wrote outside its rows"


def test_gradient_repeats_bit_for_bit():
    torch, hc = _hc()
    gen = torch.Generator(device="cuda").manual_seed(5)
    vocab, dim, count = 3000, 96, 50000
    ids = (torch.rand(count, device="cuda", generator=gen) ** 8 * vocab).long()
    x = torch.randn(count, dim, device="cuda", generator=gen)
    ws = hc.alloc_embed_workspace(vocab, dim, count)
    got = []
    for _ in range(3):
        ws.random_(0, 255)                     # what it holds on entry does not matter
        out = torch.empty(vocab, dim, device="cuda")
        hc.hc_embed_grad(x, ids, out, ws)
        got.append(out)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_workspace_for_more_ids():
    """One workspace, laid out for 2^19 + 5 ids, for any smaller number of them."""
    torch, hc = _hc()
    vocab, dim = 900, 55
    ws = hc.alloc_embed_workspace(vocab, dim, 2**19 + 5)
    gen = torch.Generator(device="cuda").manual_seed(2)
    for count in (2**19 + 5, 2**19 - 1, 171155, 85000, 20000, 8192, 700, 1):
        ids = (torch.rand(count, device="cuda", generator=gen) ** 3 * vocab).int()
        x = torch.randint(-8, 8, (count, dim), device="cuda", generator=gen).float()
        out = torch.empty(vocab, dim, device="cuda")
        hc.hc_embed_grad(x, ids, out, ws)
        want = torch.zeros(vocab, dim, device="cuda", dtype=torch.float64)
        assert torch.equal(out.double(), want.index_add(0, ids.long(), x.double())), count


def test_gradient_nan_and_infinity_stay_in_their_rows():
    torch, hc = _hc()
    x = torch.ones(6, 40, device="cuda")
    x[1, 3], x[2, 4], x[3, 5] = float("nan"), float("inf"), float("-inf")
    x[5] = float("nan")
    ids = torch.tensor([0, 1, 2, 3, 0, -1], device="cuda")
    ws = hc.alloc_embed_workspace(5, 40, 6)
    out = torch.empty(5, 40, device="cuda")
    hc.hc_embed_grad(x, ids, out, ws)
    want = torch.zeros(5, 40)
    want[0] = 2
    want[1:4] = 1
    want[1, 3], want[2, 4], want[3, 5] = float("nan"), float("inf"), float("-inf")
    assert torch.equal(out.cpu().nan_to_num(nan=9.0), want.nan_to_num(nan=9.0))
    q = torch.empty(5, 40, device="cuda", dtype=torch.int32)
    hc.hc_embed_grad(x, ids, q, ws, fixed=4.0)
    assert q[1, 3] == 0 and q[2, 4] == 2**31 - 1 and q[3, 5] == -(2**31) + 1
    assert bool((q[0] == 8).all()) and not bool(q[4].any())


def test_gradient_against_differences():
    """The lookup is linear in the table: its change along a unit step in one entry, weighted by
    dOut, is that entry's gradient.  Small whole numbers make both sides exact."""
    torch, hc = _hc()
    gen = torch.Generator().manual_seed(3)
    vocab, dim, count = 11, 6, 40
    ids = torch.randint(-1, vocab + 1, (count,), generator=gen).cuda()
    table = torch.randint(-8, 8, (vocab, dim), generator=gen).float().cuda()
    dout = torch.randint(-8, 8, (count, dim), generator=gen).float().cuda()
    ws = hc.alloc_embed_workspace(vocab, dim, count)
    grad = torch.empty(vocab, dim, device="cuda")
    hc.hc_embed_grad(dout, ids, grad, ws, scale=0.5)
    base, moved = torch.empty_like(dout), torch.empty_like(dout)
    hc.hc_embed(table, ids, base, scale=0.5)
    for v in range(vocab):
        for d in range(dim):
            step = table.clone()
            step[v, d] += 1
            hc.hc_embed(step, ids, moved, scale=0.5)
            assert float(((moved - base) * dout).double().sum()) == float(grad[v, d])


def test_other_stream_and_graph_replays():
    torch, hc = _hc()
    gen = torch.Generator(device="cuda").manual_seed(9)
    vocab, dim, count = 500, 72, 9000
    ids = torch.randint(0, vocab, (count,), device="cuda", generator=gen)
    x = torch.randn(count, dim, device="cuda", generator=gen)
    ws = hc.alloc_embed_workspace(vocab, dim, count)
    want = torch.empty(vocab, dim, device="cuda")
    hc.hc_embed_grad(x, ids, want, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(want)
    with torch.cuda.stream(side):
        hc.hc_embed_grad(x, ids, out, ws)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hc.hc_embed_grad(x, ids, out, ws)
    for k in range(4):
        x.add_(0.25 * k)
        ids.copy_((ids * 7 + k) % vocab)
        graph.replay()
        torch.cuda.synchronize()
        hc.hc_embed_grad(x, ids, want, ws)
        assert torch.equal(out, want), k


def test_rows_feed_the_coo_encode():
    """The row form in fixed point, its index expanded, is the COO encode's input: the sketch of
    the dense gradient bit for bit."""
    torch, hc = _hc()
    gen = torch.Generator(device="cuda").manual_seed(1)
    vocab, dim, count = 4000, 64, 600
    ids = torch.randint(0, vocab, (count,), device="cuda", generator=gen)
    x = torch.randn(count, dim, device="cuda", generator=gen)
    ws = hc.alloc_embed_workspace(vocab, dim, count)
    dense = torch.empty((vocab, dim), device="cuda", dtype=torch.int32)
    hc.hc_embed_grad(x, ids, dense, ws)
    rows = torch.empty(count, device="cuda", dtype=torch.int32)
    values = torch.empty((count, dim), device="cuda", dtype=torch.int32)
    touched = torch.empty(1, device="cuda", dtype=torch.int32)
    hc.hc_embed_grad_rows(x, ids, vocab, rows, values, touched, ws)
    n = int(touched)
    idx = (rows[:n, None] * dim + torch.arange(dim, device="cuda", dtype=torch.int32)).reshape(-1)
    p = hc.hc_geometry(vocab * dim, n * dim, 1.23, 1024, 5, "i32")
    y = [torch.empty(p.cells, device="cuda", dtype=torch.int32) for _ in range(2)]
    b = [torch.empty(p.words, device="cuda", dtype=torch.int32) for _ in range(2)]
    hc.hc_encode(p, dense, y[0], b[0])
    hc.hc_encode_coo(p, idx, values[:n].reshape(-1), y[1], b[1])
    assert torch.equal(y[0], y[1]) and torch.equal(b[0], b[1])


def test_binding_refusals():
    torch, hc = _hc()
    t = torch.zeros(10, 8, device="cuda")
    i = torch.zeros(4, device="cuda", dtype=torch.int32)
    ws = hc.alloc_embed_workspace(10, 8, 4)
    ok = torch.zeros(4, 8, device="cuda")
    for args in ((t, i, torch.zeros(4, 7, device="cuda")), (t, i, torch.zeros(3, 8, device="cuda")),
                 (t, i, ok.bfloat16()), (t, i.float(), ok), (t.t(), i, ok), (t, i[::2], ok[:2]),
                 (t.double(), i, ok.double()), (t[0], i, ok)):
        with pytest.raises(ValueError):
            hc.hc_embed(*args)
    for args in ((ok, i[:3], t, ws), (ok, i, torch.zeros(10, 9, device="cuda"), ws),
                 (ok.int(), i, t.double(), ws), (ok, i, t, ws.float()),
                 (ok.expand(2, 4, 8), i, t, ws)):
        with pytest.raises(ValueError):
            hc.hc_embed_grad(*args)
    with pytest.raises(hc.HCError) as e:
        hc.hc_embed_grad(ok, i, t, ws[:ws.numel() // 256 // 2 * 256])
    assert e.value.status == hc.HC_EWORKSPACE
    with pytest.raises(hc.HCError) as e:
        hc.hc_embed_grad(ok.int(), i, t, ws)
    assert e.value.status == hc.HC_EINVAL
    r, v, n = i.clone(), ok.clone(), i[:1].clone()
    with pytest.raises(ValueError):
        hc.hc_embed_grad_rows(ok, i, 10, r[:3], v, n, ws)


def test_table_of_more_dimensions():
    """A contiguous table of three dimensions is its rows: lookup and gradient take the same ones."""
    torch, hc = _hc()
    table = torch.randn(3, 5, 8, device="cuda")
    ids = torch.tensor([14, 0, 7, 14, 15, -1], device="cuda")
    rows = torch.empty(6, 8, device="cuda")
    hc.hc_embed(table, ids, rows)
    assert torch.equal(rows[:4], table.view(15, 8)[ids[:4]]) and not bool(rows[4:].any())
    want, got = torch.empty(15, 8, device="cuda"), torch.full((3, 5, 8), 7.0, device="cuda")
    ws = hc.alloc_embed_workspace(15, 8, 6)
    hc.hc_embed_grad(rows, ids, want, ws)
    assert torch.equal(want[14], rows[0] + rows[3]) and torch.equal(want[7], rows[2])
    hc.hc_embed_grad(rows, ids, got, ws)
    assert torch.equal(got.view(15, 8), want)


@pytest.mark.parametrize("vocab,dim,count,dtype", [(3000, 64, 262144 + 5, "float32"), (500, 770, 32768 + 3, "bfloat16"),
                                                   (500, 770, 32768 + 3, "float16"), (700, 768, 43691 + 9, "bfloat16"),
                                                   (50000, 3, 2**22 + 77, "float16")])
@pytest.mark.parametrize("gap,offset", [(0, 0), (3, 1)])
def test_large_lookup(vocab, dim, count, dtype, gap, offset):
    """Lookups that give every group of lanes four rows (or parts of rows), with a remainder."""
    torch, hc = _hc()
    gen = torch.Generator(device="cuda").manual_seed(dim + count)
    dt, scale = getattr(torch, dtype), 3.7
    ids = torch.randint(-vocab // 8, vocab + vocab // 8, (count,), device="cuda", generator=gen)
    ids[-1] = vocab - 1
    _, table = _strided(torch, vocab, dim, gap, offset, dt)
    table.copy_(torch.randn(vocab, dim, device="cuda", generator=gen))
    flat, out = _strided(torch, count, dim, gap, offset, dt)
    hc.hc_embed(table, ids.int(), out, scale=scale)
    valid = (ids >= 0) & (ids < vocab)
    want = (table[torch.where(valid, ids, 0)].float() * scale).to(dt)
    want[~valid] = 0
    assert torch.equal(out, want)
    out.fill_(7)
    assert bool((flat == 7).all()), "wrote outside its rows"


@pytest.mark.parametrize("vocab,dim,count", [(900, 40, 1500), (900, 40, 20000), (300, 700, 5000), (5000, 3, 70001)])
@pytest.mark.parametrize("hot", [0, 450, 899])
@pytest.mark.parametrize("x_type,g_type", [("float32", "float32"), ("float32", "int32"), ("bfloat16", "bfloat16")])
def test_rows_past_the_cap_are_not_written(vocab, dim, count, hot, x_type, g_type):
    """Fewer places than touched rows, with a frequent id (its run shared by many chunks) among the
    first, the middle and the last: the first `cap` rows are written, the count is of all."""
    torch, hc = _hc()
    hot = hot * (vocab - 1) // 899
    gen = torch.Generator().manual_seed(count + hot)
    ids = torch.randint(-3, vocab, (count,), generator=gen)
    ids[torch.rand(count, generator=gen) < 0.6] = hot
    distinct = torch.unique(ids[ids >= 0])
    n = distinct.numel()
    gt = getattr(torch, g_type)
    x, d = torch.randn(count, dim, generator=gen).to(getattr(torch, x_type)).cuda(), ids.cuda()
    ws = hc.alloc_embed_workspace(vocab, dim, count)
    dense = torch.empty((vocab, dim), device="cuda", dtype=gt)
    hc.hc_embed_grad(x, d, dense, ws)
    at = int((distinct == hot).nonzero())
    for cap in sorted({0, 1, at, at + 1, n - 1, n, n + 5}):
        rows = torch.full((n + 9,), -5, device="cuda", dtype=torch.int32)
        values = torch.full((n + 9, dim), 3, device="cuda", dtype=gt)
        touched = torch.full((1,), -1, device="cuda", dtype=torch.int32)
        hc.hc_embed_grad_rows(x, d, vocab, rows[:cap], values[:cap], touched, ws)
        k = min(cap, n)
        assert int(touched) == n
        assert torch.equal(rows[:k].cpu().long(), distinct[:k])
        assert torch.equal(values[:k], dense[distinct[:k].cuda()])
        assert bool((rows[k:] == -5).all()) and bool((values[k:] == 3).all()), cap
