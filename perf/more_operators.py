"""The dense layers' serving forms whose speed is measured: 8-bit layers, and a layer of experts for a few queries.

  quantize      s_i = max(max_k |x_ik| / 127, 2^-126), rounded to f32;  q_ik = x_ik / s_i, rounded half to even
                                                                        x [m, k], q 8-bit integers, s f32 [m]
  linear_int8   y = act(xs_i ws_j sum_k xq_ik wq_jk + b_j) + r_ij       wq [n, k] 8-bit integers, ws f32 [n]
                with xq, xs in hand ("x": "int8"), or from x in the layer's type, its rows quantized as above
  moe           p = softmax(x R^T);  the top_k experts e of a row by p, ties to the lower one;
                c_e = p_e / sum of the chosen p;  y = sum_e c_e (act(x Wg_e^T) * (x Wu_e^T)) Wd_e^T
                                                                        x [m, d], R [E, d], Wg, Wu [E, f, d], Wd [E, d, f]
                with weights in the layer's type, or 8-bit integers with an f32 scale for each of their rows

Sizes: rows, inputs and outputs are those of the dense layers beside them (workloads' batches, 26 * 64, 100 * 128,
1024 x 2816, 2048 x 5632, the ragged 777 x 1365 x 1001), the experts' numbers generic.

Keys of a case:
  op             "quantize" | "linear_int8" | "moe"
  dtype          "f32" | "f16" | "bf16": of x, biases, residual and results (of the results, where x is 8-bit)
  m, n, k        rows of x; outputs; inputs (moe: n = f, k = d)
  x              linear_int8: "int8" (quantized already) or "float"
  act            "none" | "relu" | "sigmoid" | "silu" | "gelu" (by the error function)
  bias, residual linear_int8: whether there are any
  experts, top_k moe
  weights        moe: "float" (the layer's type) or "int8"
"""
import math

import torch

own = False
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
MOST_FLOPS = 4e11              # of a drawn linear_int8; the largest listed one has 1.7e12
MOST_ELEMENTS = 1 << 28        # of a drawn case's largest matrix
MOST_WEIGHTS = 1 << 29         # of a drawn moe's experts; the largest listed one has 1.1e9


def _quantize(name, dtype, m, k):
    return {"name": name, "op": "quantize", "dtype": dtype, "m": m, "n": 0, "k": k}


def _linear(name, dtype, x, m, n, k, act, bias=True, residual=False):
    return {"name": name, "op": "linear_int8", "dtype": dtype, "x": x, "m": m, "n": n, "k": k, "act": act, "bias": bias,
            "residual": residual}


def _moe(name, dtype, weights, m, f, d, experts, top_k, act="silu"):
    return {"name": name, "op": "moe", "dtype": dtype, "weights": weights, "m": m, "n": f, "k": d, "act": act,
            "experts": experts, "top_k": top_k}


def listed():
    return [
        # the first layer's weights of a model that is loaded: 26 tables of E = 64
        _quantize("quantize_weight", "f32", 512, 1664),
        # a batch's activations, quantized once for several products; odd rows
        _quantize("quantize_ragged", "f16", 4099, 1001),
        # one query under a latency target, quantized on the way
        _linear("int8_one_query", "bf16", "float", 1, 512, 1664, "relu"),
        # a handful of queries through a wide layer: bound by reading its weights
        _linear("int8_online", "bf16", "float", 19, 8192, 4096, "silu", bias=False),
        # an inner layer with a skip connection, x quantized already
        _linear("int8_skip_layer", "bf16", "int8", 4096, 1024, 1024, "gelu", residual=True),
        # a ragged layer: nothing is a multiple of anything
        _linear("int8_ragged", "f16", "float", 777, 1365, 1001, "sigmoid"),
        # offline scoring, the largest: 100 tables of E = 128, 65536 queries (workload 5)
        _linear("int8_bulk", "bf16", "float", 65536, 1024, 12800, "relu"),
        # one query through two of eight experts: bound by latency and by reading six matrices
        _moe("moe_one_query", "bf16", "float", 1, 2816, 1024, 8, 2),
        # the same with 8-bit weights, five queries
        _moe("moe_int8_online", "bf16", "int8", 5, 2816, 1024, 8, 2),
        # a ragged layer of experts with rows that start anywhere
        _moe("moe_ragged", "f16", "float", 19, 333, 1001, 7, 3, "gelu"),
        # experts in f32
        _moe("moe_f32", "f32", "float", 8, 704, 256, 16, 4),
        # the largest: every expert of a wide layer is read for a batch of 64
        _moe("moe_batch", "bf16", "float", 64, 5632, 2048, 32, 4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "linear_int8", "linear_int8", "moe", "moe"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    even = rng.random() < 0.5   # layers are mostly sized in steps of 64

    def size(lo, hi):
        v = _log_int(rng, lo, hi)
        return -(-v // 64) * 64 if even else v

    while True:
        if op == "quantize":
            c = _quantize("", dtype, _log_int(rng, 1, 65536), size(1, 12800))
        elif op == "linear_int8":
            c = _linear("", dtype, rng.choice(["float", "int8"]), _log_int(rng, 1, 65536), size(1, 8192), size(1, 12800),
                        rng.choice(["relu", "silu", "gelu", "sigmoid", "none"]), bias=rng.random() < 0.6,
                        residual=rng.random() < 0.3)
        else:
            experts = _log_int(rng, 2, 64)
            c = _moe("", dtype, rng.choice(["float", "float", "int8"]), _log_int(rng, 1, 128), size(16, 5632), size(16, 4096),
                     experts, min(experts, rng.choice([1, 2, 2, 3, 4, 8])), rng.choice(["silu", "silu", "gelu", "relu"]))
        m, n, k = c["m"], c["n"], c["k"]
        if op == "moe":
            fits = 3 * experts * n * k <= MOST_WEIGHTS
        else:
            fits = 2.0 * m * n * k <= MOST_FLOPS and max(m * n, m * k, n * k) <= MOST_ELEMENTS
        if fits:
            del c["name"]
            return c


def _inputs(case, seed):
    """Tensors by name.  Weights keep the variance of what they multiply; rows of x are like pooled rows of trained
    tables, small values around nought, each row of a size of its own."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    m, n, k, dtype = case["m"], case["n"], case["k"], TYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dtype):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    def scales(*shape, of):
        return of * (0.5 + torch.rand(shape, device="cuda", generator=gen))

    def whole(*shape):   # 8-bit integers as quantizing normal values leaves them
        return normal(*shape, std=32.0, dtype=torch.float16).round_().clamp_(-127.0, 127.0).to(torch.int8)

    t = {}
    if case["op"] == "linear_int8" and case["x"] == "int8":
        t["x"], t["x_scale"] = whole(m, k), scales(m, of=0.5 / 32.0)
    else:
        t["x"] = normal(m, k, std=0.5)
        t["x"] *= torch.exp(normal(m, 1, std=0.5, dtype=torch.float32)).to(dtype)
    if case["op"] == "linear_int8":
        t["weight"], t["w_scale"] = whole(n, k), scales(n, of=2.0 / (32.0 * math.sqrt(k)))
        if case["bias"]:
            t["bias"] = normal(n, std=0.2)
        if case["residual"]:
            t["residual"] = normal(m, n)
    elif case["op"] == "moe":
        e = case["experts"]
        t["router"] = normal(e, k, std=2.0 / math.sqrt(k))
        for name, rows, cols in (("gate", n, k), ("up", n, k), ("down", k, n)):
            if case["weights"] == "int8":
                t["w_" + name], t["s_" + name] = whole(e, rows, cols), scales(e, rows, of=1.4 / (32.0 * math.sqrt(cols)))
            else:
                t["w_" + name] = normal(e, rows, cols, std=1.4 / math.sqrt(cols))
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


def _quantized(x):
    """(q, s): whole numbers in f32, and the scales.  The quotients are next to a border now and then: in 64 bits."""
    s = (x.abs().amax(1).double() / 127.0).float().clamp(min=2.0 ** -126)
    return torch.round(x.double() / s.double()[:, None]).clamp(-127.0, 127.0).float(), s


def _plain_moe(case, t):
    m, f, d, e, top = case["m"], case["n"], case["k"], case["experts"], case["top_k"]
    # which experts a row takes is decided by borders: in 64 bits
    p = torch.exp(torch.log_softmax(t["x"].double() @ t["router"].double().t(), 1))
    c, chosen = torch.sort(p, dim=1, descending=True, stable=True)
    c, chosen = c[:, :top], chosen[:, :top]
    c = (c / c.sum(1, keepdim=True)).float()
    x = t["x"].float()

    def weights(name, at=None):
        w = t["w_" + name] if at is None else t["w_" + name][at]
        if "s_" + name not in t:
            return w.float()
        s = t["s_" + name] if at is None else t["s_" + name][at]
        return w.float() * s[..., None]

    if m * top < e:   # few: the chosen experts' weights, one copy for each use
        at, rows = chosen.reshape(-1), x.repeat_interleave(top, 0)[:, :, None]
        h = _act(torch.bmm(weights("gate", at), rows), case["act"]) * torch.bmm(weights("up", at), rows)
        y = (torch.bmm(weights("down", at), h).view(m, top, d) * c[:, :, None]).sum(1)
    else:             # every expert for every row, and nothing of those not chosen
        share = torch.zeros(m, e, device=x.device).scatter_(1, chosen, c)
        g, u = x @ weights("gate").view(e * f, d).t(), x @ weights("up").view(e * f, d).t()
        h = (_act(g, case["act"]) * u).view(m, e, f) * share[:, :, None]
        y = h.view(m, e * f) @ weights("down").transpose(1, 2).reshape(e * f, d)
    return y.to(TYPES[case["dtype"]]), chosen.to(torch.int32), c


def _plain(case, t):
    if case["op"] == "moe":
        return _plain_moe(case, t)
    if case["op"] == "quantize":
        q, s = _quantized(t["x"])
        return q * s[:, None], s
    q, s = (t["x"].float(), t["x_scale"]) if case["x"] == "int8" else _quantized(t["x"])
    y = (q @ t["weight"].float().t()) * s[:, None] * t["w_scale"]
    if "bias" in t:
        y = y + t["bias"].float()
    y = _act(y, case["act"])
    if "residual" in t:
        y = y + t["residual"].float()
    return (y.to(TYPES[case["dtype"]]),)


# ---------------------------------------------------------------- the library's

def _own(case, t):
    import paper_2507_01676_amd as embx
    if case["op"] == "quantize":
        q, s = embx.quantize_rows(t["x"])
        return q * s[:, None], s   # (as the values that the 8 bits stand for)
    if case["op"] == "linear_int8":
        return (embx.linear_int8(t["x"], t["weight"], t["w_scale"], t.get("bias"), t.get("residual"), x_scale=t.get("x_scale"),
                                 activation=case["act"], dtype=TYPES[case["dtype"]]),)
    scales = (t["s_gate"], t["s_up"], t["s_down"]) if case["weights"] == "int8" else None
    return embx.moe_ffn(t["x"], t["router"], t["w_gate"], t["w_up"], t["w_down"], top_k=case["top_k"], scales=scales,
                        activation=case["act"], routing=True)


def run(state):
    return _own(*state) if own else _plain(*state)


def work(case):
    """Each operand read once and each result written once; two operations per product and addition of the matrix
    products (the elementwise work beside them is not counted).  Of experts, those that rows choose at random: as many
    as are expected."""
    m, n, k, size = case["m"], case["n"], case["k"], SIZES[case["dtype"]]
    if case["op"] == "quantize":
        # (the result is returned in f32, but held in 8 bits)
        return {"bytes": m * k * (size + 1) + 4 * m, "flops": 0.0}
    if case["op"] == "linear_int8":
        x = m * (k + 4) if case["x"] == "int8" else m * k * size
        return {"bytes": x + n * (k + 4) + m * n * size * (1 + case["residual"]) + (n * size if case["bias"] else 0),
                "flops": 2.0 * m * n * k}
    e, top = case["experts"], case["top_k"]
    used = e * (1.0 - (1.0 - top / e) ** m)
    weights = 3 * n * k * size if case["weights"] == "float" else 3 * n * k + 4 * (2 * n + k)
    return {"bytes": used * weights + e * k * size + 2 * m * k * size + 8 * m * top,
            "flops": 6.0 * m * top * n * k + 2.0 * m * e * k}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    t = _inputs(case, seed)
    act = {"none": lambda z: z, "relu": lambda z: z.clamp(min=0.0), "sigmoid": torch.sigmoid,
           "silu": lambda z: z * torch.sigmoid(z),
           "gelu": lambda z: z * (0.5 * torch.erfc(-z / math.sqrt(2.0)))}[case.get("act", "none")]

    def rounded(x):
        # the scale is an f32 value by definition; whole numbers are the nearest ones, even where two are as near
        s = torch.maximum((x.double().abs().max(dim=1).values / 127.0).to(torch.float32),
                          torch.tensor(2.0 ** -126, device=x.device)).double()
        v = x.double() / s.unsqueeze(1)
        low = torch.floor(v)
        up = (v - low > 0.5) | ((v - low == 0.5) & (torch.remainder(low, 2.0) == 1.0))
        return low + up.double(), s

    if case["op"] == "quantize":
        q, s = rounded(t["x"])
        return q * s.unsqueeze(1), s
    if case["op"] == "linear_int8":
        q, s = (t["x"].double(), t["x_scale"].double()) if case["x"] == "int8" else rounded(t["x"])
        y = torch.mm(q * s.unsqueeze(1), (t["weight"].double() * t["w_scale"].double().unsqueeze(1)).t())
        if "bias" in t:
            y += t["bias"].double()
        y = act(y)
        return (y + t["residual"].double() if "residual" in t else y,)
    x, top = t["x"].double(), case["top_k"]
    logits = torch.mm(x, t["router"].double().t())
    p = torch.softmax(logits, 1)
    # an expert's place: how many come before it
    before = torch.ones(case["experts"], case["experts"], device=x.device).tril(-1).bool()
    first, second = logits.unsqueeze(1), logits.unsqueeze(2)
    place = ((first > second) | ((first == second) & before)).sum(2)
    chosen = place.argsort(1)[:, :top]
    total = p.gather(1, chosen).sum(1, keepdim=True)
    y = torch.zeros_like(x)
    for e in range(case["experts"]):
        rows = (place[:, e] < top).nonzero().view(-1)
        if not len(rows):
            continue
        w = [t["w_" + name][e].double() * (t["s_" + name][e].double().unsqueeze(1) if "s_" + name in t else 1.0)
             for name in ("gate", "up", "down")]
        h = act(torch.mm(x[rows], w[0].t())) * torch.mm(x[rows], w[1].t())
        y[rows] += (p[rows, e] / total[rows, 0]).unsqueeze(1) * torch.mm(h, w[2].t())
    return y, chosen.to(torch.int32), p.gather(1, chosen) / total
