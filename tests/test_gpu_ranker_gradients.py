"""The example ranker's gradients on the GPU, each against 64 bits relative to its own norm, so that a gradient that is
missing, negated or lacks a term fails (which is shown on the reference).

Tolerance: values pass through five layers forward and back, each of which rounds to the type about three times (result,
saved sums, dz): 15 roundings of half a unit in the last place, in the worst case all of one sign and doubled by the skip
connection (TOL of test_gpu_ranker.py, with the sums' own rounding in f32).  The gradient starts from score - label: a score
rounded to the type moves it by that much of the score, hence the factor 1 + |score| / |score - label| in norms."""
import pytest

from gpu_helpers import log
from test_gpu_ranker import TOL, ranker, reference  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

MISTAKES = {"no skip gradient": {"w0", "b0", "wd", "bd"}, "no gate gradient": {"wg"}, "no up gradient": {"wu"},
            "open relu": {"w0", "b0"}}


def planted(r, q, pooled, mistake):
    """The reference's gradients with a mistake in the way back."""
    import torch
    p = {k: v.double().cpu().requires_grad_() for k, v in r.p.items()}
    dense, labels = q[2].double().cpu(), q[3].double().cpu()
    z0 = pooled.double().cpu() @ p["w0"].t() + p["b0"]
    x = (torch.relu(z0.detach()) + z0 - z0.detach()) if mistake == "open relu" else torch.relu(z0)
    x = x + torch.relu(dense @ p["wd"].t() + p["bd"])
    gate, up = torch.nn.functional.silu(x @ p["wg"].t()), x @ p["wu"].t()
    if mistake == "no gate gradient":
        gate = gate.detach()
    if mistake == "no up gradient":
        up = up.detach()
    x = (x.detach() if mistake == "no skip gradient" else x) + (gate * up) @ p["wo"].t() + p["bo"]
    z = (x @ p["ws"].t() + p["bs"]).view(-1)
    torch.nn.functional.binary_cross_entropy_with_logits(z, labels, reduction="sum").backward()
    return {k: torch.zeros_like(v) if v.grad is None else v.grad for k, v in p.items()}


def off(got, want):
    return (got.double().cpu() - want).norm().item() / want.norm().item()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("batch", [1, 100, 777])
def test_gradients_relative_to_their_norm(gpu_lib, ranker, dtype, batch):  # noqa: F811
    log(f"ranker gradients {dtype} {batch}")
    rows, E = [500, 1000, 37], 32
    r = ranker.make(rows, E, batch, dtype, width=96, inner=136)
    q = ranker.queries(rows, batch, 2, dtype)
    pooled = r.pooled(q[0], q[1], batch)
    scores, _, want = reference(r, q, pooled)
    tolerance = TOL[dtype] * (1 + (scores.norm() / (scores - q[3].double().cpu()).norm()).item())
    _, got = r.gradients(*q)
    assert set(got) == set(want)
    for name, w in want.items():
        assert off(got[name], w) <= tolerance, name
        assert tolerance < 0.5 < min(off(0 * w, w), off(-w, w))   # nothing, and the negative, would fail
    for mistake, names in MISTAKES.items():
        other = planted(r, q, pooled, mistake)
        assert max(off(other[name], want[name]) for name in names) > 2 * tolerance, mistake
