"""Views that torch negates when they are read: their memory holds other numbers than they stand for."""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu


def test_negated_views(gpu_lib):
    import torch
    log("negated views")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w, b, r = (torch.randn(*s, generator=gen, device="cuda") for s in ((6, 24), (40, 24), (40,), (6, 40)))
    f = gpu_lib
    want = f.linear(-x, w)
    column = torch.complex(x[:, :1], x[:, :1]).conj().imag   # [6, 1], minus x's first column
    for call in (lambda: f.linear(torch._neg_view(x), w), lambda: f.linear(x, torch._neg_view(w)),
                 lambda: f.linear(x, w, torch._neg_view(b)), lambda: f.linear(x, w, b, torch._neg_view(r)),
                 lambda: f.linear(x, w, out=torch._neg_view(r)), lambda: f.linear_backward(torch._neg_view(r), x, w),
                 lambda: f.gated_ffn(x, w, torch._neg_view(w)), lambda: f.linear(column, w[:, :1].contiguous())):
        with pytest.raises(ValueError, match="resolve_neg"):
            call()
    assert torch.equal(f.linear(torch._neg_view(x).resolve_neg(), w), want)
