"""The training-side operators this library is measured on, one dict a case, and how to run them.

A data-parallel step starts and ends outside the compressed aggregation: token ids are looked up in an
embedding table (lookup), the backward pass sums the output gradients of equal ids into the table's gradient
(gradient: the row-sparse input that the encode takes), and the recovered sum of a weight matrix is made
orthogonal by Newton-Schulz products before it is applied (orthogonalise).

A case's fields:
  op      "lookup", "gradient" (dense [vocab, dim]), "rows" (the touched rows alone) or "orthogonalise"
  dtype   "f32" or "bf16": the table and its lookups, the output gradient, the matrix
  lookup, gradient, rows:
    vocab, dim, count   rows and columns of the table, number of token ids
    ids     bits of a token id, 32 or 64
    masked  the share of ids that are -1 (padding: a zero row, no gradient)
    out     gradient, rows: "f32", "bf16" or "i32" (fixed point at scale 2^20)
  orthogonalise:
    batch, m, n, steps  matrices of one shape, at a stride of m * n + gap elements
    gap
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32}
FIXED = 2.0**20                          # fixed point of the int32 gradients
COEFFS = (3.4445, -4.7750, 2.0315)       # the quintic of Newton-Schulz steps
EPS = 1e-7
ZIPF = 1.1                               # token ids by rank


def _tokens(name=None, **kw):
    base = dict(op="lookup", dtype="f32", vocab=0, dim=0, count=0, ids=32, masked=0.0, out="f32")
    base.update(kw)
    if name is not None:
        base["name"] = name
    return base


def _matrix(name=None, **kw):
    base = dict(op="orthogonalise", dtype="f32", batch=1, m=0, n=0, steps=5, gap=0)
    base.update(kw)
    if name is not None:
        base["name"] = name
    return base


def listed():
    return [
        # one new token for each of sixteen sequences, BERT-base's word table: only latency counts
        _tokens("lookup_tokens_bf16", dtype="bf16", vocab=30522, dim=768, count=16),
        # a training batch of the LSTM's (33,278 words, 1500 wide): 20 streams of 35 words
        _tokens("lookup_lstm_f32", vocab=33278, dim=1500, count=700, ids=64),
        # a large batch on the 2^24 x 64 embedding table: a million lookups
        _tokens("lookup_table_f32", vocab=2**24, dim=64, count=2**20, ids=64),
        # the gradient of that LSTM batch, into the whole table's gradient
        _tokens("gradient_lstm_f32", op="gradient", vocab=33278, dim=1500, count=700, ids=64),
        # 64 sequences of 512 tokens, a tenth of them padding, into BERT-base's word table
        _tokens("gradient_bert_bf16", op="gradient", dtype="bf16", out="bf16", vocab=30522, dim=768,
                count=32768, masked=0.1),
        # the whole gradient of the 2^24 x 64 table: what the dense encode streams
        _tokens("gradient_table_f32", op="gradient", vocab=2**24, dim=64, count=2**18),
        # one worker's small batch on that table as rows, in the fixed point that the encode takes
        _tokens("rows_small_i32", op="rows", out="i32", vocab=2**24, dim=64, count=4099, ids=64),
        # a million lookups' gradient as rows
        _tokens("rows_table_f32", op="rows", vocab=2**24, dim=64, count=2**20),
        # a 3 x 3 convolution's weights, 64 of 64 channels: the smallest matrix, launches count
        _matrix("orthogonalise_conv_f32", m=64, n=576),
        # one 768 x 768 weight of each of BERT-base's twelve layers, out of the flat gradient
        _matrix("orthogonalise_bert_bf16", dtype="bf16", batch=12, m=768, n=768, gap=6498048),
        # an LSTM layer's four gates, 6000 x 1500
        _matrix("orthogonalise_lstm_f32", m=6000, n=1500),
        # VGG19's first fully connected layer, the largest matrix
        _matrix("orthogonalise_fc_bf16", dtype="bf16", m=4096, n=25088),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lookup", "gradient", "rows", "orthogonalise", "orthogonalise"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "orthogonalise":
        m, n = _log(rng, 24, 6000), _log(rng, 24, 6000)
        steps = rng.choice([4, 5, 5, 6])
        most = 2e12 / (steps * 3.0 * min(m, n) ** 2 * max(m, n))
        return _matrix(dtype=dtype, batch=max(1, min(_log(rng, 1, 16), int(most))), m=m, n=n, steps=steps,
                       gap=rng.choice([0, 0, rng.randrange(1, 5000)]))
    dim = rng.choice([64, 128, 768, _log(rng, 8, 2000), _log(rng, 8, 2000)])
    vocab = _log(rng, 1000, min(2**24, 2**29 // dim))
    count = _log(rng, 1, min(2**20, 2**26 // dim))
    out = "f32" if op == "lookup" else rng.choice(["f32", "i32"] if dtype == "f32" else ["f32", "bf16"])
    return _tokens(op=op, dtype=dtype, vocab=vocab, dim=dim, count=count, ids=rng.choice([32, 64]),
                   masked=rng.choice([0.0, 0.0, 0.1, 0.3]), out=out)


# ---- inputs ------------------------------------------------------------------------

def _ids(case, gen):
    """Zipf-ranked token ids through an odd multiplier map of the ids, some of them masked (-1)."""
    V, T = case["vocab"], case["count"]
    u = torch.rand(T, device="cuda", generator=gen, dtype=torch.float64)
    rank = (1.0 - u * (1.0 - (V + 1.0) ** (1.0 - ZIPF))) ** (1.0 / (1.0 - ZIPF))
    rank = rank.floor().clamp(1, V).to(torch.int64) - 1
    mult = 2654435761 % V | 1
    while math.gcd(mult, V) != 1:
        mult += 2
    ids = (rank * mult + 12345) % V
    if case["masked"]:
        ids = torch.where(torch.rand(T, device="cuda", generator=gen) < case["masked"], -1, ids)
    return ids.to(torch.int32 if case["ids"] == 32 else torch.int64)


def _randn(shape, std, dtype, gen):
    return (torch.randn(shape, device="cuda", generator=gen) * std).to(dtype)


def _matrices(case, gen):
    """A few strong directions over noise, as summed weight gradients have; [batch, m, n] in one flat buffer."""
    b, m, n, gap = case["batch"], case["m"], case["n"], case["gap"]
    dtype = DTYPES[case["dtype"]]
    flat = torch.zeros(b * (m * n + gap), device="cuda", dtype=dtype)
    x = flat.as_strided((b, m, n), (m * n + gap, n, 1))
    strong = min(16, m, n)
    left = torch.randn((b, m, strong), device="cuda", generator=gen)
    right = torch.randn((b, strong, n), device="cuda", generator=gen)
    x.copy_((torch.bmm(left, right) * 0.25 + torch.randn((b, m, n), device="cuda", generator=gen)) * 1e-3)
    return x


def _seeded(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 101)
    return gen


def _scale(case):
    """Lookups are scaled by sqrt(dim), as transformers with scaled embeddings do; their gradients too."""
    return float(torch.tensor(math.sqrt(case["dim"]), dtype=torch.float32))


def prepare(case, seed):
    gen, op, dtype = _seeded(seed), case["op"], DTYPES[case["dtype"]]
    st = dict(case=case)
    if op == "orthogonalise":
        st["x"] = _matrices(case, gen)
    else:
        V, D, T = case["vocab"], case["dim"], case["count"]
        st["scale"], st["tokens"] = _scale(case), _ids(case, gen)
        if op == "lookup":
            st["table"] = _randn((V, D), 0.02, dtype, gen)
        else:
            st["dout"] = _randn((T, D), 1e-3, dtype, gen)
    if own:  # the outputs and workspaces that a training program allocates once
        import paper_2402_07529_amd as hc

        def empty(*shape, dtype):
            return torch.empty(shape, device="cuda", dtype=dtype)

        if op == "orthogonalise":
            st["out"] = empty(case["batch"], case["m"], case["n"], dtype=dtype)
            st["ws"] = hc.alloc_orthogonalise_workspace(st["x"])
        elif op == "lookup":
            st["out"] = empty(T, D, dtype=dtype)
        else:
            st["ws"] = hc.alloc_embed_workspace(V, D, T)
            if op == "gradient":
                st["out"] = empty(V, D, dtype=DTYPES[case["out"]])
            else:  # what lies past the touched rows is not written
                cap = min(T, V)
                st["rows"] = torch.zeros(cap, device="cuda", dtype=torch.int32)
                st["values"] = torch.zeros((cap, D), device="cuda", dtype=DTYPES[case["out"]])
                st["touched"] = empty(1, dtype=torch.int32)
    return st


# ---- one pass ----------------------------------------------------------------------

def _plain_lookup(st):
    tokens, table = st["tokens"].long(), st["table"]
    valid = (tokens >= 0) & (tokens < table.shape[0])
    picked = table[torch.where(valid, tokens, 0)].float() * st["scale"]
    return torch.where(valid[:, None], picked, 0.0).to(table.dtype)


def _contributions(st):
    """Each token's scaled gradient: fp32, or 64-bit whole numbers of the fixed point."""
    g = st["dout"].float() * st["scale"]
    if st["case"]["out"] != "i32":
        return g
    q = torch.round(g * FIXED).nan_to_num(0.0).clamp(-2.0**31, 2.0**31)
    return q.to(torch.int64).clamp(-(2**31) + 1, 2**31 - 1)


def _narrow(total, out):
    return total.clamp(-(2**31) + 1, 2**31 - 1).to(torch.int32) if out == "i32" else total.to(DTYPES[out])


def _plain_gradient(st):
    V, D = st["case"]["vocab"], st["case"]["dim"]
    tokens, g = st["tokens"].long(), _contributions(st)
    valid = (tokens >= 0) & (tokens < V)
    total = torch.zeros((V, D), device="cuda", dtype=g.dtype)
    total.index_add_(0, tokens[valid], g[valid])
    return _narrow(total, st["case"]["out"])


def _plain_rows(st):
    V, D, T = st["case"]["vocab"], st["case"]["dim"], st["case"]["count"]
    tokens, g = st["tokens"].long(), _contributions(st)
    valid = (tokens >= 0) & (tokens < V)
    found, place = torch.unique(tokens[valid], sorted=True, return_inverse=True)
    cap = min(T, V)
    rows = torch.zeros(cap, device="cuda", dtype=torch.int32)
    rows[:found.numel()] = found.to(torch.int32)
    total = torch.zeros((cap, D), device="cuda", dtype=g.dtype)
    total.index_add_(0, place, g[valid])
    touched = torch.full((1,), found.numel(), device="cuda", dtype=torch.int32)
    return {"rows": rows, "values": _narrow(total, st["case"]["out"]), "touched": touched}


def _plain_orthogonalise(st):
    a, b, c = COEFFS
    x = st["x"].float()
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(st["case"]["steps"]):
        gram = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return (x.transpose(1, 2).contiguous() if tall else x).to(st["x"].dtype)


_PLAIN = {"lookup": _plain_lookup, "gradient": _plain_gradient, "rows": _plain_rows,
          "orthogonalise": _plain_orthogonalise}


def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return _PLAIN[op](st)
    import paper_2402_07529_amd as hc
    if op == "orthogonalise":
        hc.hc_orthogonalise(st["x"], st["out"], st["ws"], steps=case["steps"], coeffs=COEFFS, eps=EPS)
        return st["out"]
    if op == "lookup":
        hc.hc_embed(st["table"], st["tokens"], st["out"], scale=st["scale"])
        return st["out"]
    if op == "gradient":
        hc.hc_embed_grad(st["dout"], st["tokens"], st["out"], st["ws"], scale=st["scale"], fixed=FIXED)
        return st["out"]
    hc.hc_embed_grad_rows(st["dout"], st["tokens"], case["vocab"], st["rows"], st["values"], st["touched"],
                          st["ws"], scale=st["scale"], fixed=FIXED)
    return {"rows": st["rows"], "values": st["values"], "touched": st["touched"]}


# ---- what a pass cannot do without -------------------------------------------------

def _distinct(case):
    """Expected number of different valid ids."""
    V, T = case["vocab"], case["count"] * (1.0 - case["masked"])
    rank = torch.arange(1, V + 2, dtype=torch.float64) ** (1.0 - ZIPF)
    p = (rank[:-1] - rank[1:]) / (1.0 - rank[-1])
    return float((-torch.expm1(T * torch.log1p(-p.clamp(max=1 - 1e-12)))).sum())


def work(case):
    size = {"f32": 4, "bf16": 2, "i32": 4}
    if case["op"] == "orthogonalise":
        # the two products whose result is symmetric need half of their entries
        r, k, b = min(case["m"], case["n"]), max(case["m"], case["n"]), case["batch"]
        return {"bytes": 2.0 * size[case["dtype"]] * b * r * k,
                "flops": float(b * case["steps"] * (r * r * k + r**3 + 2 * r * r * k))}
    D, T, live = case["dim"], case["count"], case["count"] * (1.0 - case["masked"])
    ids = T * case["ids"] / 8
    if case["op"] == "lookup":
        return {"bytes": ids + size[case["dtype"]] * D * (_distinct(case) + T), "flops": float(live * D)}
    read = ids + size[case["dtype"]] * D * live
    if case["op"] == "gradient":
        return {"bytes": read + size[case["out"]] * D * case["vocab"], "flops": 2.0 * live * D}
    return {"bytes": read + (4 + size[case["out"]] * D) * _distinct(case), "flops": 2.0 * live * D}


# ---- the definition in 64 bits -----------------------------------------------------

def exact(case, seed):
    gen, op, dtype = _seeded(seed), case["op"], DTYPES[case["dtype"]]
    if op == "orthogonalise":
        x = _matrices(case, gen).double()
        got = []
        for y in x.unbind(0):
            y = y / (torch.linalg.vector_norm(y) + EPS)
            left = y.shape[0] <= y.shape[1]
            eye = torch.eye(min(y.shape), device="cuda", dtype=torch.float64)
            for _ in range(case["steps"]):
                g = y @ y.T if left else y.T @ y
                p = COEFFS[0] * eye + g @ (COEFFS[1] * eye + COEFFS[2] * g)
                y = p @ y if left else y @ p
            got.append(y)
        return torch.stack(got)
    V, D, T = case["vocab"], case["dim"], case["count"]
    tokens = _ids(case, gen).long()
    if op == "lookup":
        table = _randn((V, D), 0.02, dtype, gen)
        out = torch.zeros((T, D), device="cuda", dtype=torch.float64)
        at = torch.nonzero((tokens >= 0) & (tokens < V)).reshape(-1)
        out[at] = table[tokens[at]].double() * _scale(case)
        return out
    if case["out"] == "i32":  # whole numbers: compared as they are
        return None
    dout = _randn((T, D), 1e-3, dtype, gen)
    at = torch.nonzero((tokens >= 0) & (tokens < V)).reshape(-1)
    if op == "gradient":
        total = torch.zeros((V, D), device="cuda", dtype=torch.float64)
        return total.index_put_((tokens[at],), dout[at].double() * _scale(case), accumulate=True)
    seen = torch.zeros(V, device="cuda", dtype=torch.int64)
    seen[tokens[at]] = 1
    place = torch.cumsum(seen, 0) - 1
    values = torch.zeros((min(T, V), D), device="cuda", dtype=torch.float64)
    values.index_put_((place[tokens[at]],), dout[at].double() * _scale(case), accumulate=True)
    return {"rows": None, "values": values, "touched": None}
