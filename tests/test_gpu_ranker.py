"""The example ranker on the GPU: lookup and dense layers together, its scores and gradients against the same formulas
in 64 bits on the CPU, and a loss that falls."""
import importlib.util
import os

import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "ranker.py")
# Values pass through five layers, each of which rounds to the type about three times (result, saved sums, dz): 15
# roundings of half an ulp, in the worst case all of one sign and doubled by the skip connection, against the largest
# value.  f32: the sums' own rounding besides, up to 5 layers of 1664 terms at 2^-24, which is the greater part.
TOL = {"f32": 5 * 1664 * 2.0 ** -24, "f16": 30 * 2.0 ** -11, "bf16": 30 * 2.0 ** -8}


@pytest.fixture(scope="module")
def ranker():
    spec = importlib.util.spec_from_file_location("ranker_example", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(r, q, pooled):
    """(scores, loss, gradients) in 64 bits, by torch's own differentiation, from the pooled rows that the layers got."""
    import torch
    p = {k: v.double().cpu().requires_grad_() for k, v in r.p.items()}
    dense, labels = q[2].double().cpu(), q[3].double().cpu()
    x = torch.relu(pooled.double().cpu() @ p["w0"].t() + p["b0"]) + torch.relu(dense @ p["wd"].t() + p["bd"])
    x = x + (torch.nn.functional.silu(x @ p["wg"].t()) * (x @ p["wu"].t())) @ p["wo"].t() + p["bo"]
    z = (x @ p["ws"].t() + p["bs"]).view(-1)
    loss = torch.nn.functional.binary_cross_entropy_with_logits(z, labels, reduction="sum")
    loss.backward()
    return torch.sigmoid(z).detach(), loss.item() / len(labels), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("batch", [1, 100, 777])
def test_scores_and_gradients(gpu_lib, ranker, dtype, batch):
    import torch
    log(f"ranker {dtype} {batch}")
    rows, E = [500, 1000, 37], 32
    r = ranker.make(rows, E, batch, dtype, width=96, inner=136)
    q = ranker.queries(rows, batch, 2, dtype)
    pooled = r.pooled(q[0], q[1], batch)
    want, loss, grads = reference(r, q, pooled)
    got = r.scores(*q[:3])
    assert (got.double().cpu() - want).abs().max().item() <= TOL[dtype]
    assert r.plan.check_errors() == 0
    got_loss, got_grads = r.gradients(*q)
    assert abs(got_loss.item() - loss) <= TOL[dtype] * max(1.0, abs(loss))
    assert set(got_grads) == set(grads)
    for name, g in got_grads.items():
        w = grads[name]
        # against the sum of the magnitudes that a gradient is summed from: at most sqrt(batch) times the norm of its
        # parts; 1 + the largest gradient stands for it at these sizes
        scale = (1.0 + w.abs().max().item()) * max(1.0, batch ** 0.5)
        err = (g.double().cpu() - w).abs().max().item()
        assert err <= TOL[dtype] * scale, f"{name}: {err:.3e} > {TOL[dtype] * scale:.3e}"
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_loss_falls(gpu_lib, ranker, dtype):
    rows, E, batch = [500, 1000, 37], 32, 512
    r = ranker.make(rows, E, batch, dtype, width=96, inner=136)
    q = ranker.queries(rows, batch, 3, dtype)
    losses = [r.train_step(*q).item() for _ in range(40)]
    log(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
    assert losses[-1] < 0.5 * losses[0]
