"""The serving forms' Python calls: what they refuse and how, which tensors count as changed, views and shared experts."""
import pytest

import serving_reference as S
import dense_reference as R

pytestmark = pytest.mark.gpu


def operands():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    w8 = torch.randint(-127, 128, (40, 24), generator=gen, device="cuda", dtype=torch.int8)
    return dict(x=r(6, 24), w8=w8, ws=r(40).abs(), x8=w8[:6].clone(), xs=r(6).abs(), bias=r(40), res=r(6, 40), router=r(5, 24),
                gate=r(5, 40, 24), up=r(5, 40, 24), down=r(5, 24, 40))


def linear(lib, o, **kw):
    a = {**o, **kw}
    return lib.linear_int8(a["x"], a["w8"], a["ws"], a["bias"], a["res"], x_scale=a.get("x_scale"), dtype=a.get("dtype"),
                           out=a.get("out"))


def moe(lib, o, **kw):
    a = {**o, **kw}
    return lib.moe_ffn(a["x"], a["router"], a["gate"], a["up"], a["down"], top_k=a.get("top_k", 2), scales=a.get("scales"),
                       activation=a.get("activation", "silu"), out=a.get("out"))


def test_linear_int8_refusals(gpu_lib):
    import torch
    o = operands()
    linear(gpu_lib, o)
    for bad, what in (({"x": o["x"].cpu()}, "x"), ({"x": o["x"].double()}, "x"), ({"x": o["x8"]}, "x_scale"),
                      ({"x_scale": o["xs"]}, "x_scale"), ({"w8": o["w8"].float()}, "weight"), ({"w8": o["w8"][:, :8]}, "weight"),
                      ({"w8": o["w8"].t().contiguous().t()}, "weight"), ({"ws": o["ws"][:3]}, "w_scale"), ({"ws": None}, "w_scale"),
                      ({"ws": o["ws"].half()}, "w_scale"), ({"bias": o["bias"].half()}, "bias"), ({"res": o["res"][:, 1:]}, "residual"),
                      ({"dtype": torch.float16}, "dtype"), ({"dtype": "f32"}, "dtype"),
                      ({"x": o["x8"], "x_scale": o["xs"], "dtype": torch.int8}, "dtype"),
                      ({"x": o["x8"], "x_scale": o["xs"][:2]}, "x_scale"), ({"x": o["x8"], "x_scale": o["xs"], "dtype": torch.float16}, "residual"),
                      ({"out": torch.empty(6, 41, device="cuda")}, "out"), ({"out": torch.empty(6, 40, device="cuda").half()}, "out")):
        with pytest.raises(ValueError, match=what):
            linear(gpu_lib, o, **bad)
    with pytest.raises(ValueError, match="activation"):
        gpu_lib.linear_int8(o["x"], o["w8"], o["ws"], activation="tanh")
    with pytest.raises(gpu_lib.EmbxError):
        gpu_lib.linear_int8(torch.zeros(1, 131072, device="cuda"), torch.zeros(2, 131072, dtype=torch.int8, device="cuda"), o["ws"][:2])


def test_quantize_refusals(gpu_lib):
    import torch
    x = operands()["x"]
    q, s = torch.empty(6, 24, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    for bad in (x.cpu(), x.double(), x.t(), x[0], q):
        with pytest.raises(ValueError):
            gpu_lib.quantize_rows(bad)
    for out in ((q, s[:3]), (q[:3], s), (q.float(), s), (q, s.half()), (None, s), (q, None)):
        with pytest.raises(ValueError):
            gpu_lib.quantize_rows(x, out=out)


def test_moe_refusals(gpu_lib):
    import torch
    o = operands()
    moe(gpu_lib, o)
    e8 = o["gate"].to(torch.int8)
    s = torch.ones(5, 40, device="cuda")
    for bad, what in (({"x": o["x"].cpu()}, "x"), ({"router": o["router"][:, :8]}, "router"), ({"router": o["router"].half()}, "router"),
                      ({"gate": o["gate"][0]}, "w_gate"), ({"gate": o["gate"].half()}, "w_gate"), ({"up": o["up"][:4]}, "w_up"),
                      ({"down": o["gate"]}, "w_down"), ({"down": o["down"].transpose(1, 2).contiguous().transpose(1, 2)}, "w_down"),
                      ({"top_k": 0}, "top_k"), ({"top_k": 6}, "top_k"), ({"top_k": 2.0}, "top_k"), ({"activation": "tanh"}, "activation"),
                      ({"scales": (s, s, None)}, "scales"), ({"scales": (s, s, s)}, "w_gate"),
                      ({"gate": e8, "up": e8, "down": o["down"].to(torch.int8), "scales": (s, s, s)}, "scales"),
                      ({"out": torch.empty(6, 25, device="cuda")}, "out")):
        with pytest.raises(ValueError, match=what):
            moe(gpu_lib, o, **bad)


def test_gradients_are_refused(gpu_lib):
    import torch
    o = operands()
    for call, names in ((linear, ("x", "ws", "bias", "res")), (moe, ("x", "router", "gate", "up", "down"))):
        want = call(gpu_lib, o)
        for name in names:
            leaf = o[name].clone().requires_grad_()
            with pytest.raises(ValueError, match="gradient"):
                call(gpu_lib, o, **{name: leaf})
            with torch.no_grad():
                assert torch.equal(call(gpu_lib, o, **{name: leaf}), want)
    with pytest.raises(ValueError, match="gradient"):
        gpu_lib.quantize_rows(o["x"].clone().requires_grad_())
    with pytest.raises(ValueError, match="gradient"):
        linear(gpu_lib, o, out=torch.empty(6, 40, device="cuda", requires_grad=True))


def test_what_is_written_counts_as_changed(gpu_lib):
    import torch
    o = operands()
    out, y = torch.empty(6, 40, device="cuda"), torch.empty(6, 24, device="cuda")
    q, s = torch.empty(6, 24, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    before = [t._version for t in (out, y, q, s)]
    linear(gpu_lib, o, out=out), moe(gpu_lib, o, out=y), gpu_lib.quantize_rows(o["x"], out=(q, s))
    assert all(t._version > v for t, v in zip((out, y, q, s), before))
    with torch.inference_mode():
        t = torch.empty(6, 40, device="cuda")
        assert linear(gpu_lib, o, out=t) is t


def test_negated_views_are_refused(gpu_lib):
    import torch
    o = operands()
    neg = torch.complex(o["x"], o["x"]).conj().imag
    assert neg.is_neg()
    for call in (lambda: gpu_lib.quantize_rows(neg), lambda: moe(gpu_lib, o, x=neg)):
        with pytest.raises(ValueError):
            call()


def test_experts_that_share_matrices(gpu_lib):
    """Experts a stride of 0 apart, or in another order in memory."""
    import torch
    o = operands()
    one = {n: o[n][:1].expand(5, -1, -1) for n in ("gate", "up", "down")}
    want, _, _ = S.moe(o["x"], o["router"], *one.values(), 2, "silu", "f32")
    R.check(moe(gpu_lib, o, **one), want, "shared")
    mixed = torch.randn(40, 5, 24, device="cuda").transpose(0, 1)   # rows of the experts in turn
    want, _, _ = S.moe(o["x"], o["router"], mixed, o["up"], o["down"], 2, "silu", "f32")
    R.check(moe(gpu_lib, o, gate=mixed), want, "rows in turn")


def test_results_of_int8_inputs(gpu_lib):
    """Their type: dtype, or that of out, the residual or the bias, or bfloat16."""
    import torch
    o = operands()
    f = lambda **kw: gpu_lib.linear_int8(o["x8"], o["w8"], o["ws"], x_scale=o["xs"], **kw).dtype  # noqa: E731
    assert f() == torch.bfloat16 and f(dtype=torch.float16) == torch.float16 and f(bias=o["bias"]) == torch.float32
    assert f(residual=o["res"].half()) == torch.float16 and f(out=torch.empty(6, 40, device="cuda")) == torch.float32
    assert gpu_lib.linear_int8(o["x"].half(), o["w8"], o["ws"]).dtype == torch.float16
