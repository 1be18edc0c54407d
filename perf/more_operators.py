"""The layer operators this library is measured on, one dict a case, and how to run them.

Between the embedding lookup and the gradient that a data-parallel step compresses stand the layers: a matrix
product with bias, activation, dropout and residual in its epilogue (linear), its gradient, which fills most of the
flat vector that is encoded (gradient), and dropout by itself (dropout), forward or, on an output gradient,
backward.  Masks come from a counter-based generator and are stored nowhere.

A case's fields:
  op      "dropout", "linear" or "gradient"
  dtype   "f32", "bf16" or "f16": inputs and outputs
  p       the probability of a drop; 0: no dropout
  gap     elements between the rows of the inputs, beyond their columns
  residual  dropout, linear: whether a residual is added
  dropout:  m, n        rows and columns
  linear, gradient:
    m, n, k  rows (tokens), outputs, inputs of the layer
    act      "none", "relu", "gelu" (by erf), "silu", "tanh" or "sigmoid"
  linear:   bias        whether there is one
            z           whether the pre-activation is an output too, as a backward pass wants it
  gradient: out         type of the weight's and the bias's gradient
            dx          whether the input's gradient is wanted (a first layer's is not)
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ["none", "relu", "gelu", "silu", "tanh", "sigmoid"]


def _case(name=None, **kw):
    base = dict(op="linear", dtype="bf16", m=0, n=0, k=0, p=0.0, gap=0, act="none", bias=True, residual=False,
                z=False, out="f32", dx=True)
    base.update(kw)
    if name is not None:
        base["name"] = name
    return base


def listed():
    return [
        # the LSTM's dropout on a batch of 20 streams of 35 words: latency, and odd rows of 1500
        _case("dropout_lstm_f32", op="dropout", dtype="f32", m=700, n=1500, p=0.65),
        # the end of a BERT-base sub-layer, 64 sequences of 512 tokens: dropout and residual
        _case("dropout_residual_bf16", op="dropout", m=32768, n=768, p=0.1, residual=True),
        # dropout of attention weights, 64 sequences of 512 with 12 heads: the largest pass over memory
        _case("dropout_weights_f16", op="dropout", dtype="f16", m=393216, n=512, p=0.1),
        # sixteen tokens through one 768 x 768 layer: only latency counts
        _case("linear_tokens_bf16", m=16, n=768, k=768, act="gelu"),
        # a tower of NCF's perceptron on a large batch: thin, bound by memory
        _case("linear_ncf_f32", dtype="f32", m=65536, n=64, k=128, act="relu"),
        # an LSTM layer's four gates for a step's 700 words, rows that 16 bytes do not divide
        _case("linear_lstm_f32", dtype="f32", m=700, n=6000, k=1500),
        # an attention output of BERT-base with its whole epilogue
        _case("linear_bert_bf16", m=32768, n=768, k=768, p=0.1, residual=True),
        # VGG19's first fully connected layer on a large batch
        _case("linear_fc_f16", dtype="f16", m=4096, n=4096, k=25088, act="relu", p=0.5, z=True),
        # the gradient of a small classifier's head: launches count
        _case("gradient_head_f32", op="gradient", dtype="f32", m=256, n=96, k=64),
        # a BERT-base layer's, through GELU and dropout, the weight's part in the 32 bits that the encode takes
        _case("gradient_bert_bf16", op="gradient", m=32768, n=768, k=768, act="gelu", p=0.1),
        # the LSTM's output layer: 33,278 words, which 8 does not divide
        _case("gradient_words_f32", op="gradient", dtype="f32", m=700, n=33278, k=1500),
        # VGG19's first fully connected layer, the largest weight gradient
        _case("gradient_fc_bf16", op="gradient", m=4096, n=4096, k=25088, act="relu", p=0.5,
              out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dropout", "linear", "linear", "gradient", "gradient"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    gap = rng.choice([0, 0, 0, rng.randrange(1, 40)])
    if op == "dropout":
        n = rng.choice([512, 768, _log(rng, 8, 8192), _log(rng, 8, 8192)])
        return _case(op=op, dtype=dtype, m=_log(rng, 1, 2**27 // n), n=n, p=rng.choice([0.1, 0.5, 0.65]), gap=gap,
                     residual=rng.random() < 0.5)
    n = rng.choice([768, 1500, _log(rng, 8, 8192), _log(rng, 8, 8192)])
    k = rng.choice([768, 1500, _log(rng, 8, 8192), _log(rng, 8, 8192)])
    most = int(min(32768, 8e11 / (2.0 * n * k)))
    return _case(op=op, dtype=dtype, m=_log(rng, 1, most), n=n, k=k, gap=gap, act=rng.choice(ACTS),
                 p=rng.choice([0.0, 0.0, 0.1, 0.5]), bias=rng.random() < 0.8, residual=rng.random() < 0.3,
                 z=rng.random() < 0.3, out=rng.choice(["f32", dtype]), dx=rng.random() < 0.8)


# ---- inputs ------------------------------------------------------------------------

def _randn(rows, cols, std, case, gen):
    """rows x cols, with the case's gap between the rows."""
    flat = torch.zeros((rows, cols + case["gap"]), device="cuda", dtype=DTYPES[case["dtype"]])
    flat[:, :cols] = torch.randn((rows, cols), device="cuda", generator=gen) * std
    return flat[:, :cols]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 6007 + 29)
    m, n, k = case["m"], case["n"], case["k"]
    # a program's seed, and which of its draws this is (a layer, a step)
    st = dict(seed=(int(seed) * 0x9E3779B97F4A7C15 + 0x1234567) % 2**64, draw=(int(seed) * 48 + 17) % 2**40)
    if case["op"] == "dropout":
        st["x"] = _randn(m, n, 1.0, case, gen)
        if case["residual"]:
            st["residual"] = _randn(m, n, 1.0, case, gen)
        return st
    st["x"] = _randn(m, k, 1.0, case, gen)
    st["w"] = _randn(n, k, k**-0.5, case, gen)
    if case["op"] == "linear":
        if case["bias"]:
            st["bias"] = (torch.randn(n, device="cuda", generator=gen) * 0.1).to(DTYPES[case["dtype"]])
        if case["residual"]:
            st["residual"] = _randn(m, n, 1.0, case, gen)
        return st
    st["dy"] = _randn(m, n, 1e-2, case, gen)
    if case["act"] != "none":
        st["z"] = _randn(m, n, 1.0, case, gen)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if own:  # the outputs and workspaces that a training program allocates once
        import paper_2402_07529_amd as hc
        m, n, k, dtype = case["m"], case["n"], case["k"], DTYPES[case["dtype"]]

        def empty(*shape, dtype=dtype):
            return torch.empty(shape, device="cuda", dtype=dtype)

        if case["op"] == "dropout":
            st["out"] = {"y": empty(m, n)}
        elif case["op"] == "linear":
            st["out"] = {"y": empty(m, n)}
            if case["z"]:
                st["out"]["z"] = empty(m, n)
            st["ws"] = hc.alloc_linear_workspace(st["x"], st["w"])
        else:
            st["out"] = {"dw": empty(n, k, dtype=DTYPES[case["out"]]), "db": empty(n, dtype=DTYPES[case["out"]])}
            if case["dx"]:
                st["out"]["dx"] = empty(m, k)
            st["ws"] = hc.alloc_linear_grad_workspace(st["x"], st["w"])
    return st


# ---- the generator -----------------------------------------------------------------
# Philox4x32-10 (Salmon et al. 2011) with the seed as its key.  The eight elements 8 c .. 8 c + 7 of a row r share
# the call with counter (c, r, draw mod 2^32, draw div 2^32); element 8 c + e takes 16 bits of word e div 2, the low
# half first.  It is dropped where they are below T = round(65536 p); what is kept is scaled by 65536 / (65536 - T).

def _limit(p):
    return int(math.floor(p * 65536 + 0.5))


def _kept(rows, cols, p, seed, draw):
    """Truth values [rows, cols]."""
    low = 0xFFFFFFFF
    groups = (cols + 7) // 8
    row = torch.arange(rows, device="cuda", dtype=torch.int64)[:, None]
    c = [torch.arange(groups, device="cuda", dtype=torch.int64)[None, :], row,
         torch.full((1, 1), draw & low, device="cuda", dtype=torch.int64),
         torch.full((1, 1), draw >> 32, device="cuda", dtype=torch.int64)]
    key = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57  # modulo 2^64
        c = [((b >> 32) & low) ^ c[1] ^ key[0], b & low, ((a >> 32) & low) ^ c[3] ^ key[1], a & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    limit = _limit(p)
    kept = torch.empty((rows, groups, 8), device="cuda", dtype=torch.bool)
    for e in range(8):
        kept[:, :, e] = ((c[e // 2] >> (16 * (e % 2))) & 0xFFFF) >= limit
    return kept.view(rows, groups * 8)[:, :cols]


# ---- one pass ----------------------------------------------------------------------

def _drop(v, st):
    p = st["case"]["p"]
    if p == 0.0:
        return v
    return torch.where(_kept(v.shape[0], v.shape[1], p, st["seed"], st["draw"]), v * (65536.0 / (65536 - _limit(p))),
                       0.0)


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "tanh":
        return torch.tanh(z)
    if act == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi)**-0.5
    if act == "tanh":
        return 1.0 - torch.tanh(z)**2
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 - s) if act == "sigmoid" else s * (1.0 + z * (1.0 - s))


def _plain_dropout(st):
    y = _drop(st["x"].float(), st)
    if "residual" in st:
        y = y + st["residual"].float()
    return {"y": y.to(st["x"].dtype)}


def _plain_linear(st):
    dtype = st["x"].dtype
    z = torch.matmul(st["x"].float(), st["w"].float().t())
    if "bias" in st:
        z = z + st["bias"].float()
    y = _drop(_act(z, st["case"]["act"]), st)
    if "residual" in st:
        y = y + st["residual"].float()
    out = {"y": y.to(dtype)}
    if st["case"]["z"]:
        out["z"] = z.to(dtype)
    return out


def _plain_gradient(st):
    case = st["case"]
    dz = _drop(st["dy"].float(), st)
    if case["act"] != "none":
        dz = dz * _act_slope(st["z"].float(), case["act"])
    kind = DTYPES[case["out"]]
    out = {"dw": torch.matmul(dz.t(), st["x"].float()).to(kind), "db": dz.sum(0).to(kind)}
    if case["dx"]:
        out["dx"] = torch.matmul(dz, st["w"].float()).to(st["x"].dtype)
    return out


_PLAIN = {"dropout": _plain_dropout, "linear": _plain_linear, "gradient": _plain_gradient}


def run(st):
    case = st["case"]
    if not own:
        return _PLAIN[case["op"]](st)
    import paper_2402_07529_amd as hc
    out, rand = st["out"], dict(p=case["p"], seed=st["seed"], draw=st["draw"])
    if case["op"] == "dropout":
        hc.hc_dropout(st["x"], out["y"], residual=st.get("residual"), **rand)
    elif case["op"] == "linear":
        hc.hc_linear(st["x"], st["w"], out["y"], st["ws"], bias=st.get("bias"), residual=st.get("residual"),
                     z=out.get("z"), act=case["act"], **rand)
    else:
        hc.hc_linear_grad(st["dy"], st["ws"], x=st["x"], w=st["w"], z=st.get("z"), dx=out.get("dx"), dw=out["dw"],
                          db=out["db"], act=case["act"], **rand)
    return out


# ---- what a pass cannot do without -------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    s, m, n, k = size[case["dtype"]], case["m"], case["n"], case["k"]
    if case["op"] == "dropout":
        return {"bytes": float(s * m * n * (3 if case["residual"] else 2)), "flops": float(m * n)}
    if case["op"] == "linear":
        rows = 1 + case["residual"] + case["z"]
        return {"bytes": float(s * (m * k + n * k + m * n * rows + n * case["bias"])), "flops": 2.0 * m * n * k}
    read = m * k + m * n * (1 if case["act"] == "none" else 2) + (n * k + m * k if case["dx"] else 0)
    return {"bytes": float(s * read + size[case["out"]] * (n * k + n)),
            "flops": 2.0 * m * n * k * (2 if case["dx"] else 1)}


# ---- the definition in 64 bits -----------------------------------------------------

def _times(const, v):
    """The high and low 32 bits of const * v, from products of 16 bits."""
    c1, c0, v1, v0 = const >> 16, const & 0xFFFF, v >> 16, v & 0xFFFF
    low = c0 * v0
    mid = c1 * v0 + (low >> 16)
    mid2 = c0 * v1 + (mid & 0xFFFF)
    return c1 * v1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)


def _factors(case, inputs):
    """What dropout multiplies each element by, in 64 bits, a block of rows at a time."""
    m, n, limit = case["m"], case["n"], _limit(case["p"])
    if limit == 0:
        return torch.ones((1, 1), device="cuda", dtype=torch.float64)
    out = torch.empty((m, n), device="cuda", dtype=torch.float64 if m * n < 2**26 else torch.float32)
    groups, step = (n + 7) // 8, max(1, 2**24 // n)
    which = torch.arange(n, device="cuda")
    for r0 in range(0, m, step):
        r1 = min(m, r0 + step)
        shape = (r1 - r0, groups)
        x0 = torch.arange(groups, device="cuda").expand(shape)
        x1 = torch.arange(r0, r1, device="cuda")[:, None].expand(shape)
        x2, x3 = torch.full_like(x0, inputs["draw"] % 2**32), torch.full_like(x0, inputs["draw"] // 2**32)
        for i in range(10):
            k0 = (inputs["seed"] % 2**32 + i * 0x9E3779B9) % 2**32
            k1 = (inputs["seed"] // 2**32 + i * 0xBB67AE85) % 2**32
            h0, l0 = _times(0xD2511F53, x0)
            h1, l1 = _times(0xCD9E8D57, x2)
            x0, x1, x2, x3 = h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0
        words = torch.stack([x0, x1, x2, x3], 2).view(r1 - r0, groups * 4)[:, which // 2]
        out[r0:r1] = torch.where((words // 65536 ** (which % 2)) % 65536 < limit, 0.0, 1.0)
    return out


def exact(case, seed):
    st = _inputs(case, seed)
    factor, scale = _factors(case, st), 65536.0 / (65536 - _limit(case["p"]))
    if case["op"] == "dropout":
        y = torch.empty((case["m"], case["n"]), device="cuda", dtype=torch.float64)
        torch.mul(st["x"], factor, out=y)
        y *= scale
        if case["residual"]:
            y += st["residual"]
        return {"y": y}
    act, x, w = case["act"], st["x"].double(), st["w"].double()
    if case["op"] == "linear":
        z = torch.mm(x, w.T)
        if case["bias"]:
            z += st["bias"].double()
        a = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0),
             "gelu": lambda: 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0)),
             "silu": lambda: z * torch.special.expit(z), "tanh": lambda: torch.tanh(z),
             "sigmoid": lambda: torch.special.expit(z)}[act]()
        y = a * factor * scale
        if case["residual"]:
            y = y + st["residual"].double()
        return {"y": y, "z": z} if case["z"] else {"y": y}
    g = st["dy"].double() * factor * scale
    if act != "none":
        z = st["z"].double()
        sg = torch.special.expit(z)
        g = g * {"relu": lambda: torch.where(z > 0, 1.0, 0.0),
                 "gelu": lambda: (0.5 * torch.special.erfc(-z / math.sqrt(2.0))
                                  + z / math.sqrt(2.0 * math.pi) * torch.exp(-z * z / 2.0)),
                 "silu": lambda: sg + z * sg * torch.special.expit(-z), "tanh": lambda: 1.0 / torch.cosh(z)**2,
                 "sigmoid": lambda: sg * torch.special.expit(-z)}[act]()
    out = {"dw": torch.mm(g.T, x), "db": g.sum(0)}
    if case["dx"]:
        out["dx"] = torch.mm(g, w)
    return out
