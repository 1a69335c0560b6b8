"""A tensor given as ``out`` counts as changed: torch refuses to differentiate through a value of it that is gone."""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["linear", "gated_ffn"])
@pytest.mark.parametrize("save", [False, True])
def test_out_counts_as_changed(gpu_lib, name, save):
    import torch
    log(f"{name} {save}")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w, out = (torch.randn(*s, generator=gen, device="cuda") for s in ((6, 24), (40, 24), (6, 40)))

    def call(out):
        if name == "linear":
            gpu_lib.linear(x, w, out=out, save=save)
        else:
            gpu_lib.gated_ffn(x, w, w, out=out, save=save)

    before = out._version
    call(out)
    assert out._version == before + 1
    big = torch.zeros(8, 50, device="cuda")
    call(big[1:7, 2:42])
    assert big._version == 1
    leaf = torch.ones(6, 40, device="cuda", requires_grad=True)
    product = (leaf * out).sum()   # saves out
    call(out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.backward()
    with pytest.raises(ValueError):
        call(out[:5])
    version = out._version
    with torch.inference_mode():   # tensors made there have no version
        call(torch.empty(6, 40, device="cuda"))
        call(out)
    assert out._version == version + 1
    assert x._version == 0 and w._version == 0
