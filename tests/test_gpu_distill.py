"""Distillation from a teacher's top logits on the GPU against the definition in 64 bits, on the
host.  Tolerances count roundings (see `bounds`)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1412_1576_amd import operators
    return operators


def reference(x, ids, t, tau, log_norm=None, weight=None):
    """(loss, gradient, q, P, |terms|) of the definition; x, t float64 arrays of the values the tensors
    hold, weight None: ones."""
    with np.errstate(all="ignore"):
        N, V = x.shape
        loss, grad = np.zeros(N), np.zeros((N, V))
        qs, ps, sizes = np.zeros((N, V)), np.zeros((N, V)), np.zeros(N)
        for i in range(N):
            w = 1.0 if weight is None else weight[i]
            y = x[i] / tau
            m = y.max()
            e = np.exp(y - (m if m > -np.inf else 0.0))
            q = e / e.sum() if e.sum() != 0 else e
            log_q = y - (m if m > -np.inf else 0.0) - np.log(e.sum())
            log_q = np.where(np.isneginf(x[i]), -np.inf, log_q)
            full = (ids[i] >= 0) & (ids[i] < V)
            at, tt = ids[i][full].astype(np.int64), t[i][full] / tau
            if log_norm is None:
                top = tt.max() if len(tt) and tt.max() > -np.inf else 0.0
                s = np.exp(tt - top).sum()
                lp = tt - top - (np.log(s) if s != 0 else 0.0)
            else:
                lp = tt - log_norm[i]
            p = np.exp(lp)
            r, others = 0.0, np.setdiff1d(np.arange(V), at)
            if log_norm is not None and len(others):
                r = max(0.0, 1.0 - p.sum()) / len(others)
            P = np.zeros(V)
            P[others] = r
            np.add.at(P, at, p)
            mass = P.sum()
            qs[i], ps[i] = q, P
            if mass == 0 or w == 0:
                continue
            term = [pj * (l - log_q[a]) for pj, l, a in zip(p, lp, at) if pj != 0]
            even = r * (np.log(r) - log_q[others]) if r > 0 else np.zeros(0)
            loss[i] = tau * tau * (np.sum(term) + even.sum())
            if np.isnan(e.sum()) or np.isnan(mass):
                loss[i] = np.nan
            sizes[i] = sum(pj * (abs(l) + abs(log_q[a])) for pj, l, a in zip(p, lp, at) if pj != 0)
            sizes[i] += np.abs(even).sum()
            grad[i] = w * tau * (mass * q - P)
    return loss, grad, qs, ps, sizes


U = 2.0 ** -24


def bounds(x, tau, sizes, q, P, weight, dtype, out):
    """Roundings.  exp2((S - m) c): its argument is rounded twice and c once, 3 U of |y|, the result 2 U;
    sums of 32 bits inside a thread add at most V / 256 + 32 times (a thread has a 256th of a
    row, or less), every one U; the masses p are rounded once; weights and scales four times.  In the loss the
    terms of the sum e count with their share q; in the gradient T w (M q - P) what q is off by counts M = sum P
    times (M > 1 where a norm is too small for its slots)."""
    V = x.shape[1]
    with np.errstate(all="ignore"):
        y = np.abs(x - x.max(1, keepdims=True)) / tau
        y = np.where(q > 0, y, 0.0)
        log_s = (q * (3 * y + 2)).sum(1) * U + (V / 256 + 32) * U
        loss = tau * tau * (np.maximum(P.sum(1), 1.0) * log_s + 2 * U * sizes) + 1e-30
        rel = (3 * y + 8) * U + log_s[:, None]
        w = np.ones(len(x)) if weight is None else np.abs(weight)
        mq = P.sum(1, keepdims=True) * q
        grad = w[:, None] * tau * (mq * rel + 8 * U * (P + mq))
        # an exponential below the smallest normal number of 32 bits keeps fewer bits or is 0: off by that number
        # at most, times T w M / s with s >= 1 (the base of the sum is one of its logits)
        grad = grad + w[:, None] * tau * np.maximum(P.sum(1, keepdims=True), 1.0) * 2.0 ** -126
        half = torch.finfo(dtype).eps / 2
        # (half a step below the smallest normal number too)
        grad = grad + np.abs(out) * half * 1.01 + torch.finfo(dtype).smallest_normal * 2 * half
    # a row of NaN that counts all the same has exact zeros
    return np.nan_to_num(loss, nan=0.0, posinf=np.inf), np.nan_to_num(grad, nan=0.0, posinf=np.inf)


def compare(got, want, bound, what):
    got, want = got.astype(np.float64), np.asarray(want, np.float64)
    odd = ~np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[odd & ~np.isnan(want)], want[odd & ~np.isnan(want)]), what
    off = np.abs(got[~odd] - want[~odd]) - np.broadcast_to(bound, want.shape)[~odd]
    assert off.size == 0 or off.max() <= 0, (what, off.max())


def make(N, V, k, dtype, seed, pad=0, offset=0, tdtype=torch.float32, scale=3.0):
    """(logits, ids, teacher) on the GPU; rows pad elements apart beyond V, the first offset elements in."""
    g = torch.Generator().manual_seed(seed)
    store = torch.full((N * (V + pad) + offset + 8,), 777.0).to(dtype)
    x = store[offset:offset + N * (V + pad)].view(N, V + pad)[:, :V]
    x.copy_((torch.randn(N, V, generator=g) * scale).to(dtype))
    x = store.cuda()[offset:offset + N * (V + pad)].view(N, V + pad)[:, :V]
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(N)])
    if k > V:
        ids = torch.cat([ids, torch.full((N, k - V), -1)], 1)
    t = (torch.randn(N, k, generator=g) * 2 + 1).to(tdtype)
    return x, ids.cuda(), t.cuda()


def host(x):
    return None if x is None else x.detach().double().cpu().numpy()


def check(ops, x, ids, t, tau=1.0, log_norm=None, weight=None, both=True):
    """All three calls against the definition."""
    xr, ir, tr, nr, wr = host(x), ids.cpu().numpy(), host(t), host(log_norm), host(weight)
    tau32 = float(np.float32(tau))
    loss, grad, q, P, sizes = reference(xr, ir, tr, tau32, nr, wr)
    lb, gb = bounds(xr, tau32, sizes, q, P, wr, x.dtype, grad)
    got, g = ops.distill_loss_and_grad(x, ids, t, temperature=tau, log_norm=log_norm, weight=weight)
    assert g.dtype == x.dtype and g.shape == x.shape and got.dtype == torch.float32
    compare(got.cpu().numpy(), loss, lb, "loss of the step")
    compare(host(g), grad, gb, "gradient of the step")
    if not both:
        return
    whole = reference(xr, ir, tr, tau32, nr)[0]
    lb = bounds(xr, tau32, reference(xr, ir, tr, tau32, nr)[4], q, P, wr, x.dtype, grad)[0]
    leaf = x.detach().requires_grad_(True)
    got = ops.distill_loss(leaf, ids, t, temperature=tau, log_norm=log_norm)
    up = torch.ones_like(got) if weight is None else weight
    g, = torch.autograd.grad(got, leaf, up)
    compare(got.detach().cpu().numpy(), whole, lb, "loss")
    compare(host(g), grad, gb, "gradient")
    with torch.no_grad():
        again = ops.distill_loss(x, ids, t, temperature=tau, log_norm=log_norm)
    assert torch.equal(again.isnan(), got.isnan()) and torch.equal(again.nan_to_num(0), got.detach().nan_to_num(0))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N,V,k", [(1, 1, 1), (3, 7, 9), (2, 63, 5), (5, 64, 64), (4, 257, 1), (3, 1000, 16),
                                   (2, 4099, 256), (2, 20_011, 1024), (70, 515, 0), (1100, 130, 12)])
def test_sizes(ops, N, V, k, dtype):
    check(ops, *make(N, V, k, TYPES[dtype], seed=V + k), tau=1.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,k", [(1, 1, 1), (3, 7, 9), (4, 257, 1), (3, 4099, 256), (70, 515, 0), (1100, 130, 12),
                                   (2, 12, 12)])
def test_sizes_with_a_floor(ops, N, V, k, dtype):
    x, ids, t = make(N, V, k, TYPES[dtype], seed=V + k)
    full = torch.where(ids >= 0, t.double(), -torch.inf)
    norm = torch.logsumexp(full, 1) + torch.rand(N).cuda() if k else torch.zeros(N).cuda()
    check(ops, x, ids, t, log_norm=norm.float())
    # a norm too small for the slots: more mass than 1, no floor
    check(ops, x, ids, t, log_norm=norm.float() - 2.0)


@pytest.mark.parametrize("N,V", [(1, 141_043), (3, 100_003), (1, 1_000_003), (300, 30_011)])
@pytest.mark.parametrize("rest", [False, True])
def test_long_rows(ops, N, V, rest):
    x, ids, t = make(N, V, 50, torch.bfloat16, seed=N)
    norm = (torch.logsumexp(t.double(), 1) + 0.3).float() if rest else None
    n = min(N, 4)   # the definition takes its time
    check(ops, x[:n], ids[:n], t[:n], tau=2.0, log_norm=None if norm is None else norm[:n])
    loss, grad = ops.distill_loss_and_grad(x, ids, t, temperature=2.0, log_norm=norm)
    some, part = ops.distill_loss_and_grad(x[:n], ids[:n], t[:n], temperature=2.0,
                                           log_norm=None if norm is None else norm[:n])
    assert torch.allclose(loss[:n], some, rtol=1e-5, atol=1e-5)
    assert torch.allclose(grad[:n].float(), part.float(), rtol=0.01, atol=1e-6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 0), (5, 3), (2000, 1)])
def test_rows_that_start_anywhere(ops, pad, offset, dtype):
    x, ids, t = make(5, 1003, 20, TYPES[dtype], seed=pad, pad=pad, offset=offset)
    check(ops, x, ids, t)
    x, ids, t = make(3, 20_003, 20, TYPES[dtype], seed=pad, pad=pad, offset=offset)
    check(ops, x, ids, t)


@pytest.mark.parametrize("stride", [1003, 1004, 1500])
@pytest.mark.parametrize("start", [0, 1, 7])
def test_gradient_rows_that_start_elsewhere(ops, stride, start):
    """Through the C entry: gradient rows aligned otherwise than the logits', and what lies between
    them as it was."""
    import ctypes as C
    from paper_1412_1576_amd import lda
    N, V = 4, 1003
    x, ids, t = make(N, V, 20, torch.bfloat16, seed=3)
    loss, want = ops.distill_loss_and_grad(x, ids, t)
    store = torch.full((N * stride + 16,), 5.0, dtype=torch.bfloat16, device="cuda")
    r = ops._distill_rows(x, ids, t, 1.0, None)
    L = lda.load_library()
    need = L.lda_distill_workspace(C.byref(r))
    w = ops._workspace(r, need, x.device)
    assert L.lda_distill_step(C.byref(r), loss.data_ptr(), store.data_ptr() + 2 * start, stride) == 0
    torch.cuda.synchronize()
    rows = store[start:start + N * stride].view(N, stride)
    assert torch.equal(rows[:, :V], want)
    assert (rows[:, V:] == 5.0).all() and (store[:start] == 5.0).all() and (store[start + N * stride:] == 5.0).all()
    del w


def test_types_of_the_teacher(ops):
    for tdtype in TYPES.values():
        for itype in (torch.int32, torch.int64):
            x, ids, t = make(6, 700, 33, torch.float32, seed=4, tdtype=tdtype)
            check(ops, x, ids.to(itype), t)
    # wider rows of the teacher's tensors
    x, ids, t = make(6, 700, 33, torch.float32, seed=4)
    check(ops, x, ids[:, :20], t[:, :20])
    check(ops, x[::2], ids[::2], t[::2])


@pytest.mark.parametrize("rest", [False, True])
def test_ids_twice_and_outside(ops, rest):
    x, ids, t = make(6, 50, 12, torch.float32, seed=5)
    ids[0, :] = 7                       # all the same
    ids[1, 3] = ids[1, 9]               # twice
    ids[2, :4] = torch.tensor([-1, 50, 1 << 40, -(1 << 40)], device="cuda")
    t[2, :4] = torch.tensor([float("nan"), float("inf"), 1e38, -1e38])
    ids[3, :] = -1                      # no teacher
    t[4, :6] = -float("inf")            # slots without mass
    t[5, :] = -float("inf")             # none with any
    norm = torch.full((6,), 4.5, device="cuda") if rest else None
    if rest:
        t.clamp_(max=2.0)
    check(ops, x, ids, t, log_norm=norm)


def test_masked_and_odd_logits(ops):
    inf, low = float("inf"), torch.finfo(torch.float32).min
    x, ids, t = make(12, 130, 6, torch.float32, seed=6)
    ids = torch.arange(6, device="cuda").expand(12, 6).contiguous()
    x[0, 60:] = -inf
    x[1, 60:] = low
    x[2, :] = low                       # a row that a mask of the lowest value leaves nothing
    x[3, :] = -inf                      # and one of -inf
    x[4, 2] = -inf                      # the teacher has mass where the student has none
    x[5, 99] = float("nan")
    x[6, 99] = inf
    x[7, :] = torch.finfo(torch.float32).max
    x[8, 99] = 1e30
    x[9, :] = -inf
    x[9, 3] = 1.0                       # one class is left
    x[10, 99] = float("nan")
    ids[10] = -1                        # a row without a teacher, whatever the logits hold
    x[11, 2], t[11, 2] = -inf, -inf     # masked on both sides
    check(ops, x, ids, t)
    check(ops, x, ids, t, tau=0.25)
    check(ops, x.bfloat16()[[0, 3, 4, 5, 6, 9, 10, 11]], ids[[0, 3, 4, 5, 6, 9, 10, 11]], t[[0, 3, 4, 5, 6, 9, 10, 11]])
    rows = [0, 3, 4, 5, 6, 9]
    norm = torch.full((12,), 5.0, device="cuda")
    check(ops, x[rows], ids[rows], t[rows].clamp(max=2.5), log_norm=norm[rows])
    # -inf only where a slot without mass is: the floor's classes are all there
    y = torch.randn(2, 40, device="cuda")
    y[0, 2] = -inf
    u = t[:2].clamp(max=2.0).clone()
    u[0, 2] = -inf
    check(ops, y, ids[:2], u, log_norm=norm[:2])


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("V,times", [(3000, 1), (10_001, 1), (20_001, 1), (30_001, 1), (30_001, 6), (60_003, 11)])
def test_masked_and_odd_logits_of_longer_rows(ops, V, times, rest):
    """The same through a workgroup's registers of every shape, and through slices; masks that leave a
    slice, or all but one, without anything."""
    inf, low = float("inf"), torch.finfo(torch.float32).min
    x, ids, t = make(10, V, 6, torch.float32, seed=V)
    ids = torch.tensor([0, 1, 2, V // 2, V - 2, V - 1], device="cuda").expand(10, 6).contiguous()
    x[0, : V // 2] = low
    x[1, 10:] = low
    x[2, :] = low
    x[3, :] = -inf
    x[4, 2] = -inf
    x[5, V // 3] = float("nan")
    x[6, V - 7] = inf
    x[7, 20: V - 20] = -inf
    x[8, :] = -inf
    x[8, V // 2] = 1.0
    x[9, V // 5] = float("nan")
    ids[9] = -1
    t.clamp_(max=2.0)
    norm = torch.full((10,), 4.0, device="cuda") if rest else None
    if times == 1:
        check(ops, x, ids, t, log_norm=norm)
        return
    # more rows take another kernel: the rows are those of the first ten
    want = ops.distill_loss_and_grad(x, ids, t, log_norm=norm)
    got = ops.distill_loss_and_grad(x.repeat(times, 1), ids.repeat(times, 1), t.repeat(times, 1),
                                    log_norm=None if norm is None else norm.repeat(times))
    for g, w in zip(got, want):
        g, w = g.view(times, *w.shape), w.expand(times, *w.shape)
        assert torch.equal(g.isnan(), w.isnan()) and torch.equal(g.isinf(), w.isinf())
        some = torch.isfinite(w)
        assert torch.allclose(g[some], w[some], rtol=1e-5, atol=1e-7)


def test_weights(ops):
    x, ids, t = make(9, 300, 10, torch.float32, seed=7)
    x[2] = float("nan")
    w = torch.randn(9, device="cuda")
    w[2] = w[5] = 0.0
    check(ops, x, ids, t, weight=w, both=False)
    wide = torch.zeros(9, 3, device="cuda")
    wide[:, 1] = w
    loss, grad = ops.distill_loss_and_grad(x, ids, t, weight=w)
    for other in (wide[:, 1], w.clone()):
        l2, g2 = ops.distill_loss_and_grad(x, ids, t, weight=other)
        assert torch.equal(loss, l2) and torch.equal(grad, g2)
    assert (loss[[2, 5]] == 0).all() and (grad[[2, 5]] == 0).all()
    one = torch.full((1,), 0.5, device="cuda").expand(9)
    check(ops, x[3:], ids[3:], t[3:], weight=one[3:])


def test_broadcast_and_strided_upstream(ops):
    x, ids, t = make(8, 500, 10, torch.float32, seed=8)
    leaf = x.requires_grad_(True)
    for reduce, weight in ((lambda l: l.sum(), 1.0), (lambda l: l.mean(), 1 / 8), (lambda l: l[::2].sum(), None)):
        g, = torch.autograd.grad(reduce(ops.distill_loss(leaf, ids, t)), leaf)
        w = torch.full((8,), weight, device="cuda") if weight else torch.tensor([1.0, 0.0] * 4, device="cuda")
        want = ops.distill_loss_and_grad(x, ids, t, weight=w)[1]
        assert torch.equal(g, want)
    up = torch.randn(8, 2, device="cuda")
    g, = torch.autograd.grad(ops.distill_loss(leaf, ids, t), leaf, up[:, 0])
    assert torch.equal(g, ops.distill_loss_and_grad(x, ids, t, weight=up[:, 0].contiguous())[1])
    # an expanded input: the gradients of its copies add up
    row = torch.randn(1, 500, device="cuda", requires_grad=True)
    ops.distill_loss(row.expand(8, 500), ids, t).sum().backward()
    each = ops.distill_loss_and_grad(row.detach().expand(8, 500), ids, t)[1]
    assert torch.allclose(row.grad[0], each.sum(0), rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("rest", [False, True])
def test_gradient_against_differences(ops, rest):
    """(loss(S + h d) - loss(S - h d)) / 2h along directions of length 1.  Only T^2 M log sum exp(S / T)
    is not linear in S; its third derivative along d is T^2 M times the third central moment of d_v / T,
    numbers within sqrt(2) / T of each other, so at most 0.0963 * 2.83 / T = 0.136 for T = 2, M = 1: h = 1/8 is
    off by h^2 / 6 * 0.136 = 3.6e-4 at most.  Losses below 32 are good to 2^-19 (see `bounds`): 2 * 2^-19 / 2h =
    1.6e-5 more."""
    x, ids, t = make(4, 60, 6, torch.float32, seed=9, scale=1.0)
    norm = (torch.logsumexp(t.double() / 2, 1) + 0.5).float() if rest else None
    kw = {"temperature": 2.0, "log_norm": norm}
    grad = ops.distill_loss_and_grad(x, ids, t, **kw)[1]
    h = 0.125
    for seed in range(5):
        d = torch.randn(4, 60, generator=torch.Generator().manual_seed(seed)).cuda()
        d /= d.norm(dim=1, keepdim=True)
        up, down = ops.distill_loss(x + h * d, ids, t, **kw), ops.distill_loss(x - h * d, ids, t, **kw)
        slope = ((up - down) / (2 * h)).cpu()
        assert up.max() < 32
        assert ((grad * d).sum(1).cpu() - slope).abs().max() <= 4e-4


def test_the_binding_refuses(ops):
    x, ids, t = make(4, 100, 5, torch.float32, seed=10)
    bad = [dict(logits=x.double()), dict(logits=x[0]), dict(logits=x.t()), dict(ids=ids.short()),
           dict(ids=ids[:3]), dict(teacher=t[:, :4]), dict(teacher=t.cpu()), dict(teacher=t.clone().requires_grad_()),
           dict(log_norm=torch.zeros(3, device="cuda")), dict(log_norm=torch.zeros(4, device="cuda").double()),
           dict(log_norm=torch.zeros(1, device="cuda").expand(4)), dict(logits=x[:, :0])]
    for change in bad:
        kw = {"logits": x, "ids": ids, "teacher": t, **change}
        with pytest.raises(ValueError):
            ops.distill_loss(**kw)
        with pytest.raises(ValueError):
            ops.distill_loss_and_grad(**kw)
    with pytest.raises(ValueError):
        ops.distill_loss_and_grad(x, ids, t, weight=torch.ones(3, device="cuda"))
    from paper_1412_1576_amd.lda import LdaError
    for tau in (0.0, -1.0, float("nan"), 1e9):
        with pytest.raises(LdaError, match="temperature"):
            ops.distill_loss(x, ids, t, temperature=tau)
    with pytest.raises(LdaError, match="1024"):
        ops.distill_loss(x, ids.repeat(1, 300), t.repeat(1, 300))
    # and no rows are no work
    loss, grad = ops.distill_loss_and_grad(x[:0], ids[:0], t[:0])
    assert loss.shape == (0,) and grad.shape == (0, 100)
    y = x[:0].requires_grad_(True)
    ops.distill_loss(y, ids[:0], t[:0]).sum().backward()
    assert y.grad.shape == (0, 100)


def test_other_streams_and_two_calls_at_once(ops):
    big = make(40, 200_003, 30, torch.bfloat16, seed=11)
    small = make(64, 5_003, 30, torch.float32, seed=12)
    want = [ops.distill_loss_and_grad(*big), ops.distill_loss_and_grad(*small)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, data in zip(streams, (big, small)):
            with torch.cuda.stream(s):
                got.append(ops.distill_loss_and_grad(*data))
        torch.cuda.synchronize()
        for (l, g), (lw, gw) in zip(got, want):
            assert torch.equal(l, lw) and torch.equal(g, gw)


@pytest.mark.parametrize("N,V", [(3, 100_003), (1100, 515)])
def test_captured_and_replayed(ops, N, V):
    x, ids, t = make(N, V, 20, torch.bfloat16, seed=13)
    w = torch.rand(N, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ops.distill_loss_and_grad(x, ids, t, weight=w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        loss, grad = ops.distill_loss_and_grad(x, ids, t, weight=w)
        alone = ops.distill_loss(x, ids, t)
    for i in range(4):
        x.copy_(torch.randn(N, V, generator=torch.Generator().manual_seed(i)).to(x.dtype))
        w.uniform_()
        graph.replay()
        torch.cuda.synchronize()
        lw, gw = ops.distill_loss_and_grad(x, ids, t, weight=w)
        assert torch.equal(loss, lw) and torch.equal(grad, gw) and torch.equal(alone, lw)
        x.add_(1.0).sum()


def test_the_backward_captured(ops):
    x, ids, t = make(5, 60_011, 20, torch.float32, seed=14)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        leaf = x.clone().requires_grad_(True)
        torch.autograd.grad(ops.distill_loss(leaf, ids, t).mean(), leaf)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        loss = ops.distill_loss(leaf, ids, t)
        grad, = torch.autograd.grad(loss.mean(), leaf)
    w = torch.full((5,), 0.2, device="cuda")
    for i in range(3):
        with torch.no_grad():
            leaf.copy_(x * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        lw, gw = ops.distill_loss_and_grad(leaf.detach(), ids, t, weight=w)
        assert torch.equal(loss.detach(), lw) and torch.equal(grad, gw)


@pytest.mark.parametrize("tau", [1 / 1024, 0.05, 30.0, 1024.0])
@pytest.mark.parametrize("rest", [False, True])
def test_temperatures(ops, tau, rest):
    x, ids, t = make(5, 3001, 40, torch.float32, seed=15)
    norm = None
    if rest:
        norm = (torch.logsumexp(t.double() / tau, 1) + 0.4).float()
        # (a norm of thousands is itself good to 2^-24 of that only: the masses are those of the float)
    check(ops, x, ids, t, tau=tau, log_norm=norm)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("V,k", [(100, 1024), (1000, 1000), (3000, 700), (30_000, 1024)])
def test_many_slots_of_few_classes(ops, V, k, rest):
    """More slots than threads, most classes several times, some slots empty."""
    x, ids, t = make(3, V, min(k, V), torch.float32, seed=16)
    g = torch.Generator().manual_seed(V)
    ids = torch.randint(-20, min(V, 300) + 20, (3, k), generator=g).cuda()
    t = torch.randn(3, k, generator=g).cuda()
    full = torch.where((ids >= 0) & (ids < V), t.double(), -torch.inf)
    norm = (torch.logsumexp(full, 1) + 0.3).float() if rest else None
    check(ops, x, ids, t, log_norm=norm)


def test_lazily_negated_tensors_are_refused(ops):
    """The imaginary part of a conjugated tensor is a view whose memory holds the opposite numbers."""
    x, ids, t = make(4, 100, 5, torch.float32, seed=17)
    weight = torch.ones(4, dtype=torch.complex64, device="cuda").conj().imag
    assert weight.is_neg()
    with pytest.raises(ValueError, match="resolve_neg"):
        ops.distill_loss_and_grad(x, ids, t, weight=weight)
    loss, grad = ops.distill_loss_and_grad(x, ids, t, weight=weight.resolve_neg())
    assert (loss == 0).all() and (grad == 0).all()
