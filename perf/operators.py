"""The dense layers whose speed is measured: what a recommender has the library do once its rows are pooled.

The pooled rows of a batch, [queries, tables * E], go through fully connected layers and gated feed-forward
blocks; a model in training goes back through them.  Four operators, in f32, f16 and bf16:

  linear       z = x W^T + b,  y = act(z) + r          x [m, k], W [n, k], b [n], r [m, n]
  linear_grad  dz = dy * act'(z),  dx = dz W,  dW = dz^T x,  db = column sums of dz
  gated        g = x Wg^T + bg,  u = x Wu^T + bu,  h = act(g) * u
  gated_grad   dg = dh * u * act'(g),  du = dh * act(g),  dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x,
               dbg, dbu = column sums of dg, du

The gradients take z (or g and u) as the forward pass has saved them, in the layer's type.

Sizes come from the repository's five workloads: their batches (one query up to 65536) are m, their tables times
E (26 * 64, 26 * 128, 100 * 128) are k of a first layer; n and the inner layers are generic.

Keys of a case:
  op, dtype      as above; "f32" | "f16" | "bf16"
  m, n, k        rows of x, outputs, inputs
  act            "none" | "relu" | "sigmoid" | "silu" | "gelu" (by the error function)
  bias           with a bias (its gradient is an output too)
  residual       linear: a residual is added after the activation
  save           linear, gated: z, or g and u, are outputs too, as in a training step
"""
import math

import torch

own = False
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
MOST_FLOPS = 4e11          # a drawn case's; the largest listed case has 1.7e12
MOST_ELEMENTS = 1 << 28    # of a drawn case's largest matrix


def _case(name, op, dtype, m, n, k, act, bias=True, residual=False, save=False):
    return {"name": name, "op": op, "dtype": dtype, "m": m, "n": n, "k": k, "act": act, "bias": bias,
            "residual": residual, "save": save}


def listed():
    return [
        # one query under a latency target: the first layer over 26 tables of E = 64
        _case("first_layer_one_query", "linear", "bf16", 1, 512, 1664, "relu"),
        # the last layer: one score a query (batch of workload 2)
        _case("score", "linear", "f16", 2048, 1, 256, "sigmoid"),
        # the dense features' first layer: an odd, tiny k; bound by what it writes
        _case("dense_features", "linear", "f16", 16384, 512, 13, "relu"),
        # an inner layer with a skip connection, in training (z is kept)
        _case("skip_layer", "linear", "bf16", 4096, 1024, 1024, "gelu", residual=True, save=True),
        # the pooled rows as the lookup leaves them, in f32 (batch of workload 4)
        _case("first_layer_f32", "linear", "f32", 4096, 512, 1664, "relu"),
        # offline scoring, the largest: 100 tables of E = 128, 65536 queries (workload 5)
        _case("first_layer_bulk", "linear", "bf16", 65536, 1024, 12800, "relu"),
        # a training step's way back through the first layer (workload 3: 26 tables of E = 128)
        _case("first_layer_grad", "linear_grad", "f16", 16384, 1024, 3328, "relu"),
        # an odd small layer trained in f32
        _case("small_layer_grad_f32", "linear_grad", "f32", 3001, 77, 200, "silu"),
        # a handful of queries through a gated block: bound by reading its weights
        _case("gated_online", "gated", "bf16", 19, 2816, 1024, "silu", bias=False),
        # a gated block over a full batch
        _case("gated_bulk", "gated", "bf16", 16384, 5632, 2048, "silu", bias=False),
        # a gated block in training, its forward pass's g and u given
        _case("gated_grad", "gated_grad", "bf16", 8192, 4096, 1024, "silu", bias=False),
        # a ragged gated block with biases and another activation
        _case("gated_grad_ragged", "gated_grad", "f16", 777, 1365, 1001, "gelu"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear_grad", "gated", "gated_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    while True:
        m, n, k = _log_int(rng, 1, 65536), _log_int(rng, 1, 8192), _log_int(rng, 1, 12800)
        if rng.random() < 0.5:   # layers are mostly sized in steps of 64
            n, k = -(-n // 64) * 64, -(-k // 64) * 64
        c = _case("", op, dtype, m, n, k, rng.choice(["relu", "silu", "gelu", "sigmoid", "none"]),
                  bias=rng.random() < 0.6, residual=op == "linear" and rng.random() < 0.3,
                  save=op in ("linear", "gated") and rng.random() < 0.3)
        if work(c)["flops"] <= MOST_FLOPS and max(m * n, m * k, n * k) <= MOST_ELEMENTS:
            del c["name"]
            return c


def _inputs(case, seed):
    """Tensors by name.  Weights keep the variance of what they multiply; rows of x are like pooled rows of trained
    tables: small values around nought."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    m, n, k, dtype = case["m"], case["n"], case["k"], TYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    t = {"x": normal(m, k, std=0.5)}
    gated = case["op"].startswith("gated")
    for name in (("w_gate", "w_up") if gated else ("weight",)):
        t[name] = normal(n, k, std=2.0 / math.sqrt(k))
    if case["op"] in ("linear", "gated"):
        for name in (("b_gate", "b_up") if gated else ("bias",)):
            t[name] = normal(n, std=0.2) if case["bias"] else None
        t["residual"] = normal(m, n) if case["residual"] else None
    else:
        t["dy"] = normal(m, n, std=0.1)
        for name in (("g", "u") if gated else ("z",)):
            t[name] = normal(m, n)
    return t


def prepare(case, seed):
    return case, _inputs(case, seed)


# ---------------------------------------------------------------- the plain form

def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, act):
    """act'(z)"""
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 - s)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _affine(x, w, b):
    z = x @ w.t()
    return z if b is None else z + b


def _plain(case, t):
    dtype, act = TYPES[case["dtype"]], case["act"]
    f = {name: None if v is None else v.to(torch.float32) for name, v in t.items()}
    if case["op"] == "linear":
        z = _affine(f["x"], f["weight"], f["bias"])
        y = _act(z, act)
        if f["residual"] is not None:
            y = y + f["residual"]
        out = (y, z) if case["save"] else (y,)
    elif case["op"] == "gated":
        g, u = _affine(f["x"], f["w_gate"], f["b_gate"]), _affine(f["x"], f["w_up"], f["b_up"])
        h = _act(g, act) * u
        out = (h, g, u) if case["save"] else (h,)
    elif case["op"] == "linear_grad":
        dz = f["dy"] * _slope(f["z"], act)
        out = (dz @ f["weight"], dz.t() @ f["x"])
        if case["bias"]:
            out += (dz.sum(0),)
    else:
        dg, du = f["dy"] * f["u"] * _slope(f["g"], act), f["dy"] * _act(f["g"], act)
        out = (dg @ f["w_gate"] + du @ f["w_up"], dg.t() @ f["x"], du.t() @ f["x"])
        if case["bias"]:
            out += (dg.sum(0), du.sum(0))
    return tuple(v.to(dtype) for v in out)


# ---------------------------------------------------------------- the library's

def _own(case, t):
    import paper_2507_01676_amd as embx
    op, act = case["op"], case["act"]
    if op == "linear":
        out = embx.linear(t["x"], t["weight"], t["bias"], t["residual"], activation=act, save=case["save"])
    elif op == "gated":
        out = embx.gated_ffn(t["x"], t["w_gate"], t["w_up"], t["b_gate"], t["b_up"], activation=act, save=case["save"])
    elif op == "linear_grad":
        out = embx.linear_backward(t["dy"], t["x"], t["weight"], t["z"], activation=act, bias=case["bias"])
    else:
        out = embx.gated_ffn_backward(t["dy"], t["x"], t["w_gate"], t["w_up"], t["g"], t["u"], activation=act,
                                      bias=case["bias"])
    return out if isinstance(out, tuple) else (out,)


def run(state):
    return _own(*state) if own else _plain(*state)


def work(case):
    """Each operand read once and each result written once; two operations per product and addition of the matrix
    products (the elementwise work beside them is not counted)."""
    m, n, k = case["m"], case["n"], case["k"]
    mats = 2 if case["op"].startswith("gated") else 1
    weights = mats * n * k
    if case["op"].endswith("_grad"):
        # dy, saved values, x and W read; dx, dW and db written
        elements = m * n * (1 + mats) + 2 * m * k + 2 * weights + (mats * n if case["bias"] else 0)
        flops = 4.0 * m * n * k * mats
    else:
        elements = m * k + weights + m * n * (1 + case["residual"] + (mats if case["save"] else 0)) \
            + (mats * n if case["bias"] else 0)
        flops = 2.0 * m * n * k * mats
    return {"bytes": elements * (4 if case["dtype"] == "f32" else 2), "flops": flops}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    v = {name: t.double() for name, t in _inputs(case, seed).items() if t is not None}
    act = case["act"]

    def sigma(z):
        return torch.sigmoid(z)

    def phi(z):   # the normal distribution function
        return 0.5 * torch.erfc(-z / math.sqrt(2.0))

    value = {"none": lambda z: z, "relu": lambda z: z.clamp(min=0.0), "sigmoid": sigma,
             "silu": lambda z: z * sigma(z), "gelu": lambda z: z * phi(z)}[act]
    slope = {"none": lambda z: torch.ones_like(z), "relu": lambda z: (z > 0).double(),
             "sigmoid": lambda z: sigma(z) * sigma(-z),
             "silu": lambda z: sigma(z) + z * sigma(z) * sigma(-z),
             "gelu": lambda z: phi(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)}[act]

    def affine(w, b):
        return torch.addmm(v[b], v["x"], v[w].t()) if b in v else torch.mm(v["x"], v[w].t())

    if case["op"] == "linear":
        z = affine("weight", "bias")
        y = value(z) + v["residual"] if "residual" in v else value(z)
        return (y, z) if case["save"] else (y,)
    if case["op"] == "gated":
        g, u = affine("w_gate", "b_gate"), affine("w_up", "b_up")
        return (value(g) * u, g, u) if case["save"] else (value(g) * u,)
    if case["op"] == "linear_grad":
        dz = v["dy"] * slope(v["z"])
        out = [torch.mm(dz, v["weight"]), torch.mm(dz.t(), v["x"])]
        sums = [dz]
    else:
        dg, du = v["dy"] * v["u"] * slope(v["g"]), v["dy"] * value(v["g"])
        out = [torch.mm(dg, v["w_gate"]) + torch.mm(du, v["w_up"]), torch.mm(dg.t(), v["x"]), torch.mm(du.t(), v["x"])]
        sums = [dg, du]
    return tuple(out + ([s.sum(0) for s in sums] if case["bias"] else []))
