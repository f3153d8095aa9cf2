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


def taken_out(x, ids, P, tau):
    """What classes with a slot may leave behind that are summed with the others and taken out again (logits above
    -64, or -1024 in long rows): each 7 roundings, of a sum of 8 differences from the base, which is at most 12 / T
    below the largest logit."""
    off = np.zeros(len(x))
    for i in range(len(x)):
        at = np.unique(ids[i][(ids[i] >= 0) & (ids[i] < x.shape[1])])
        others = np.setdiff1d(np.arange(x.shape[1]), at)
        near = x[i][(x[i] > -1100) & (x[i] < 1100)]
        if len(others) and len(near):
            off[i] = tau * P[i][others[0]] * len(at) * 7 * 8 * (near.max() - near.min() + 12) * 2.0 ** -24
    return off


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
    if norm is not None:
        lb = lb + np.nan_to_num(taken_out(xr, ids[rows].cpu().numpy(), P, tau))
    # (a loss above the largest number of 32 bits is rounded to infinity: T times a mask of the lowest value may be)
    want = np.where(want > np.finfo(np.float32).max, np.inf, want)
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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [-1e9, -1e30, None])
@pytest.mark.parametrize("shape", SHAPES)
def test_masked_classes_with_a_slot(ops, shape, mask, dtype):
    """A teacher's largest logits where it has fewer classes than slots: what it and the student mask has a slot, and
    no mass.  Only the classes without a slot count beside the slots."""
    n, v = sizes(shape, dtype)
    low = torch.finfo(TYPES[dtype]).min
    mask = low if mask is None else mask
    x, ids, t = make(n, v, 16, TYPES[dtype], seed=2)
    x.scatter_(1, ids[:, 8:], mask)
    t[:, 8:] = -float("inf")
    x[1].scatter_(0, ids[1, 12:], low)             # two kinds of masks
    x[2, (ids[2, 0] + 1) % v] = -float("inf")
    t[2, 15] = 1.0                                 # masked by the student alone
    x[3, : v // 2] = mask                          # also classes without a slot: a large loss
    for tau in (1.0, 2.0, 4.0):
        full = t.double() / tau
        norm = (torch.logsumexp(full, 1) + 0.3).float()
        compare_rows(ops, x, ids, t, [0, 1, 2, 3, n - 1], tau, norm)


@pytest.mark.parametrize("mask", [-50.0, -80.0, -1000.0, -1050.0, -1e5])
@pytest.mark.parametrize("n,v,k", [(3, 20, 16), (3, 300, 200), (3, 2_000, 1_000), (3, 15_000, 1_000), (2, 90_001, 1_000)])
def test_most_classes_have_a_slot_and_a_mask(ops, n, v, k, mask):
    """Masks around the borders, in every place of a chunk; and rows of logits that all lie below the borders."""
    x, ids, t = make(n, v, k, torch.float32, seed=3)
    x.scatter_(1, ids[:, k // 8:], mask)
    t[:, k // 8:] = -float("inf")
    norm = (torch.logsumexp(t.double(), 1) + 0.5).float()
    compare_rows(ops, x, ids, t, list(range(n)), 1.0, norm)
    compare_rows(ops, x - 70.0, ids, t, list(range(n)), 1.0, norm)
    compare_rows(ops, x - 1500.0, ids, t, list(range(n)), 1.0, norm)


@pytest.mark.parametrize("k", [1, 3, 4, 70])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_norm_of_no_mass(ops, shape, k):
    """The log-sum of a row of empty slots, or of logits of -infinity, is -infinity: no slot has mass, and the
    floor is 1 / (classes without a slot)."""
    n, v = shape
    x, ids, t = make(n, v, k, torch.float32, seed=4)
    norm = (torch.logsumexp(t.double(), 1) + 0.3).float()
    ids[0] = -1
    ids[1, 0] = v                      # one slot and its like outside the classes
    ids[1, 1:] = -5
    t[1] = float("nan")                # not looked at
    t[2] = -float("inf")               # slots that name their classes, without mass
    norm[:3] = -float("inf")
    held = norm.clone()
    held[:3] = 0.0                     # (any norm gives the same)
    got = compare_rows(ops, x, ids, t, [0, 1, 2, 3, n - 1], 1.0, norm, held)
    assert all(torch.isfinite(g).all() for g in sum(got, ()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_infinite_mass(ops, shape, dtype):
    """A teacher's logit of +infinity, with a norm as without one, or a norm of -infinity beside a logit: the row is not a
    number; and with weight 0 it is left out like any other."""
    n, v = sizes(shape, dtype)
    x, ids, t = make(n, v, 8, TYPES[dtype], seed=5)
    norm = (torch.logsumexp(t.double(), 1) + 0.3).float()
    t[0, 3] = float("inf")
    t[1, 3], norm[1] = float("inf"), float("inf")
    norm[2] = -float("inf")
    odd = torch.zeros(n, dtype=torch.bool, device="cuda")
    for z in (norm, None):
        odd[:3] = True
        odd[2] = z is not None
        leaf = x.detach().requires_grad_(True)
        loss = ops.distill_loss(leaf, ids, t, log_norm=z)
        grad, = torch.autograd.grad(loss, leaf, torch.ones_like(loss))
        for l, g in ((loss, grad), ops.distill_loss_and_grad(x, ids, t, log_norm=z)):
            assert torch.equal(l.isnan(), odd) and torch.isfinite(l[~odd]).all()
            assert torch.equal(g.isnan().any(1), odd) and torch.equal(g.isnan().all(1), odd)
        left = ops.distill_loss_and_grad(x, ids, t, log_norm=z, weight=(~odd).float())
        assert torch.isfinite(left[0]).all() and (left[0][odd] == 0).all() and (left[1][odd] == 0).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_what_several_slots_of_a_class_change(ops, tau, rest):
    """Against one slot with the mass of all: the gradient is the same, and the loss less by
    T^2 sum of p log(P / p).  In 64 bits that is exact; each side is good to 1e-6 of numbers below 10 (`bounds`)."""
    n, v, k = 5, 700, 40
    x, ids, t = make(n, v, k, torch.float32, seed=6)
    ids[:, 1::2] = ids[:, ::2]
    norm = (torch.logsumexp(t.double() / tau, 1) + (0.2 if rest else 0.0)).float()
    once = (tau * torch.logaddexp(t[:, ::2].double() / tau, t[:, 1::2].double() / tau)).float()
    p = torch.exp(t.double() / tau - norm.double()[:, None])
    both = (p[:, ::2] + p[:, 1::2]).repeat_interleave(2, 1)
    less = tau * tau * (p * torch.log(both / p)).sum(1)
    z = norm if rest else None
    loss, grad = ops.distill_loss_and_grad(x, ids, t, temperature=tau, log_norm=z)
    want, same = ops.distill_loss_and_grad(x, ids[:, ::2].contiguous(), once, temperature=tau, log_norm=z)
    assert less.min() > 0.01   # (much more than the sides may be off)
    assert ((want.double() - loss.double()) - less).abs().max() < 4e-5
    assert (grad - same).abs().max() < 4e-6


def test_the_shapes_are_all_there_are():
    """SHAPES against the table of the source: each of its rows is chosen by one, and slices by one."""
    import os
    import re
    from paper_1412_1576_amd import build
    text = open(os.path.join(build.CSRC, "distill.hip")).read()
    table = re.search(r"kShapes\[\] = \{(.*)\};", text).group(1)
    table = [tuple(map(int, row.split(","))) for row in re.findall(r"\{([^{}]*)\}", table)]
    chosen = []
    for n, v in SHAPES:
        fits = [s for s in table if v // 4 <= s[0] * s[1]]
        chosen.append(fits[0] if fits and (fits[0][0] < 1024 or n >= fits[0][2]) else None)
    assert chosen == table + [None]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_odd_logits_in_every_shape(ops, shape, rest, dtype):
    """The rows of a batch that takes the shape, each against the definition: masks that leave a thread, or all but one,
    nothing, numbers that are none, a row without a teacher."""
    inf = float("inf")
    n, v = sizes(shape, dtype)
    n = max(n, 13)
    x, ids, t = make(n, v, 6, TYPES[dtype], seed=7)
    low = torch.finfo(x.dtype).min
    ids[:] = torch.tensor([0, 1, 2, v // 2, v - 2, v - 1], device="cuda")
    x[0, : v // 2] = low
    x[1, 10:] = low
    x[2, :] = low
    x[3, :] = -inf
    x[4, 2] = -inf
    x[5, v // 3] = float("nan")
    x[6, v - 7] = inf
    x[7, 20: v - 20] = -inf
    x[8, :] = -inf
    x[8, v // 2] = 1.0
    x[9, v // 5] = float("nan")
    ids[9] = -1
    x[10, 2], t[10, 2] = -inf, -inf
    t.clamp_(max=2.0)
    norm = torch.full((n,), 4.0, device="cuda") if rest else None
    if rest:
        ids[9] = torch.arange(6, device="cuda")
        t[9], norm[9] = -inf, inf       # a floor alone
        x[9] = x[11]
    compare_rows(ops, x, ids, t, list(range(12)) + [n - 1], 1.0, norm)
