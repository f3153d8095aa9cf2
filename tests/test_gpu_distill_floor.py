"""Distillation with a floor (a log-normaliser) where classes are masked, and rows of the teacher that are
empty or odd, through every form that a row can take; against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from test_gpu_distill import TYPES, bounds, compare, host, make, ops, reference

pytestmark = pytest.mark.gpu

# rows and 32-bit classes (twice as many of 16 bits) for which a row is held by 64, 256 (two sizes) or 1024 threads
# (three sizes, the longer two from 64 and 128 rows on), or is cut into slices
SHAPES = [(4, 1_000), (4, 3_000), (4, 10_001), (4, 20_001), (66, 30_001), (130, 60_003), (4, 90_001)]


def sizes(shape, dtype):
    n, v = shape
    return n, v if dtype == "f32" else 2 * v


def compare_rows(ops, x, ids, t, rows, tau=1.0, log_norm=None, held=None):
    """The step, and loss and gradient through autograd, of all rows; `rows` of them against the definition.
    held: the norms for the definition, where they differ."""
    got = [ops.distill_loss_and_grad(x, ids, t, temperature=tau, log_norm=log_norm)]
    leaf = x.detach().requires_grad_(True)
    loss = ops.distill_loss(leaf, ids, t, temperature=tau, log_norm=log_norm)
    got.append((loss.detach(), torch.autograd.grad(loss, leaf, torch.ones_like(loss))[0]))
    with torch.no_grad():
        alone = ops.distill_loss(x, ids, t, temperature=tau, log_norm=log_norm)
    assert torch.equal(alone.nan_to_num(0.25), loss.detach().nan_to_num(0.25))
    norm = log_norm if held is None else held
    xr = host(x[rows])
    want, grad, q, P, size = reference(xr, ids[rows].cpu().numpy(), host(t[rows]), tau, host(None if norm is None else norm[rows]))
    lb, gb = bounds(xr, tau, size, q, P, None, x.dtype, grad)
    for what, (loss, g) in zip(("step", "autograd"), got):
        compare(loss[rows].cpu().numpy(), want, lb, "loss, " + what)
        compare(host(g[rows]), grad, gb, "gradient, " + what)
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tau", [1.0, 2.0, 4.0])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2], SHAPES[-1]])
def test_masks_of_the_lowest_value_beside_the_slots(ops, shape, tau, dtype):
    """T^2 sum of r (S - m) / T is a number of 32 bits; sums of a few (S - m) / T in 32 bits are not."""
    n, v = sizes(shape, dtype)
    x, ids, t = make(n, v, 16, TYPES[dtype], seed=1)
    x[:, :v // 10] = torch.finfo(x.dtype).min   # neighbours, which a thread adds
    x.scatter_(1, ids, 0.5)
    norm = (torch.logsumexp(t.double() / tau, 1) + 0.05).float()
    got = compare_rows(ops, x, ids, t, list(range(n)), tau, norm)
    assert all(torch.isfinite(loss).all() and (loss > 1e35).all() for loss, _ in got)
