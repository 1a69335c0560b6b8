"""The dense layers and torch's differentiation: the calls record no gradients, and say so instead of leaving them out; what
they write over is known to have changed."""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu


def tensors():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w, b, r = (torch.randn(*s, generator=gen, device="cuda") for s in ((6, 24), (40, 24), (40,), (6, 40)))
    return x, w, b, r


CALLS = {"linear": lambda f, x, w, b, r: f.linear(x, w, b, r),
         "linear_backward": lambda f, x, w, b, r: f.linear_backward(r, x, w),
         "gated_ffn": lambda f, x, w, b, r: f.gated_ffn(x, w, w, b),
         "gated_ffn_backward": lambda f, x, w, b, r: f.gated_ffn_backward(r, x, w, w, r, r)}


@pytest.mark.parametrize("name", CALLS)
def test_operands_that_require_a_gradient(gpu_lib, name):
    import torch
    log(name)
    given = {"linear": (0, 1, 2, 3), "gated_ffn": (0, 1, 2)}.get(name, (0, 1, 3))
    for at in given:
        t = list(tensors())
        want = CALLS[name](gpu_lib, *t)
        t[at].requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            CALLS[name](gpu_lib, *t)
        with pytest.raises(ValueError, match="gradient"):   # of a graph, not a leaf
            t[at] = t[at] * 1.0
            CALLS[name](gpu_lib, *t)
        for off in (torch.no_grad(), torch.inference_mode()):
            with off:
                got = CALLS[name](gpu_lib, *t)
            for g, v in zip(got if isinstance(got, tuple) else (got,), want if isinstance(want, tuple) else (want,)):
                assert g is v is None or (torch.equal(g, v) and not g.requires_grad)
        t[at] = t[at].detach()
        assert CALLS[name](gpu_lib, *t) is not None


def test_out_that_requires_a_gradient(gpu_lib):
    import torch
    x, w, b, r = tensors()
    out = torch.empty_like(r).requires_grad_()
    for call in (lambda: gpu_lib.linear(x, w, out=out), lambda: gpu_lib.gated_ffn(x, w, w, out=out)):
        with pytest.raises(ValueError, match="gradient"):
            call()


def test_inside_a_function_of_autograd(gpu_lib):
    """As a layer that torch differentiates: the calls in forward and backward of a torch.autograd.Function."""
    import torch

    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, z = gpu_lib.linear(x, w, b, activation="silu", save=True)
            ctx.save_for_backward(x, w, z)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w, z = ctx.saved_tensors
            return gpu_lib.linear_backward(dy.contiguous(), x, w, z, activation="silu")

    x, w, b, r = tensors()
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    (Linear.apply(*leaves) * r).sum().backward()
    again = [t.double().clone().requires_grad_() for t in (x, w, b)]
    (torch.nn.functional.silu(again[0] @ again[1].t() + again[2]) * r.double()).sum().backward()
    for p, q in zip(leaves, again):   # sums of 40 products at most, in 32 bits
        torch.testing.assert_close(p.grad.double(), q.grad, rtol=1e-5, atol=1e-5)
