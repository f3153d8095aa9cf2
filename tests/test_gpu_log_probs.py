"""Log probabilities of tokens, entropy, top alternatives and gradients on the GPU against the definition in 64 bits.
Tolerances count roundings (see `check`); ids are equal."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24
INF = float("inf")


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1412_1576_amd import operators
    return operators


def make(n, v, dtype, seed, pad=0, offset=0, scale=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    store = torch.full((n * (v + pad) + offset + 8,), 777.0, device="cuda").to(dtype)
    x = store[offset:offset + n * (v + pad)].view(n, v + pad)[:, :v]
    x.copy_((torch.randn(n, v, generator=g, device="cuda") * scale).to(dtype))
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    return x, t


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert torch.equal(got.isnan(), want.isnan()), what
    odd = ~torch.isfinite(want)
    assert torch.equal(got[odd & ~want.isnan()], want[odd & ~want.isnan()]), what
    off = ((got - want).abs() - bound)[~odd]
    assert off.numel() == 0 or off.max() <= 0, (what, float(off.max()))


def definition(x, t, tau):
    """(log_prob, entropy, log p, p, |y|, log s) in 64 bits, y = (S - largest) / T, s = sum e^y"""
    y = x.double() / tau
    m = y.amax(1, keepdim=True)
    odd = y.isnan().any(1, keepdim=True) | (m == INF)
    y = y - torch.where(m == -INF, 0.0, m)
    s = y.exp().sum(1, keepdim=True)
    none = s == 0
    log_p = torch.where(none, -INF, y - s.log())
    p = log_p.exp()
    term = torch.where(p > 0, p * log_p, 0.0)
    entropy = -term.sum(1)
    given = (t >= 0) & (t < x.shape[1])
    log_prob = torch.where(given, log_p.gather(1, t.clamp(0, x.shape[1] - 1)[:, None].long())[:, 0], 0.0)
    log_prob = torch.where(odd[:, 0] & given, torch.nan, log_prob)
    entropy = torch.where(odd[:, 0], torch.nan, entropy)
    return log_prob, entropy, log_p, p, torch.where(p > 0, y.abs(), 0.0), torch.where(none, 0.0, s.log()), odd, given


def best(x, k):
    """Ids of the k largest above -infinity, equal ones by class, and -1."""
    value, ids = torch.sort(x.float() + 0.0, dim=1, descending=True, stable=True)
    value, ids = value[:, :k], torch.where(value == -INF, -1, ids)[:, :k]
    if k > ids.shape[1]:
        ids = torch.nn.functional.pad(ids, (0, k - ids.shape[1]), value=-1)
    return ids


def check(ops, x, t, tau=1.0, top=0, gradient=True, seed=0):
    """An exponential of the running form: its argument is rounded three times, the result is good to 2 U; each rise
    of the base by at least 1.38 multiplies once more, with an argument as large as the rise; the base lies within 1.4
    of the largest in the end: (10 |y| + 24) U of the term in all.  A thread adds at most V / 256 + 16 terms, some 24
    joins follow.  The entropy has terms of size y + 2 in place of 1, and their roundings."""
    n, v = x.shape
    tau = float(torch.tensor(tau, dtype=torch.float32))
    want_lp, want_h, log_p, p, y, log_s, odd, given = definition(x, t, tau)
    adds = v / 256 + 40
    q = p.nan_to_num(0.0)
    es = (q * (10 * y + 24)).sum(1) * U + adds * U
    eh = es + ((q * (y + 2) * (20 * y + 60)).sum(1) + 2 * adds * (q * (y + 2)).sum(1)) * U
    ls = log_s[:, 0].abs().nan_to_num(0.0)
    eh = eh + U * (ls + want_h.abs().nan_to_num(0.0))
    out = ops.token_log_probs(x, t, temperature=tau, top=top)
    assert all(o.dtype == torch.float32 for o in out[:2])
    elp = es + U * (ls + want_lp.abs().nan_to_num(0.0, posinf=0.0))
    close(out[0], want_lp, elp, "log_prob")
    close(out[1], want_h, eh, "entropy")
    assert not (out[1] < 0).any()
    if top:
        ids, values = out[2:]
        assert ids.dtype == torch.int32 and values.dtype == torch.float32 and ids.shape == values.shape == (n, top)
        want = torch.where(odd, -1, best(x, top))
        assert torch.equal(ids.long(), want)
        lp = torch.where(want >= 0, log_p.gather(1, want.clamp(min=0)), -INF)
        lp = torch.where(odd, torch.nan, lp)
        close(values, lp, es[:, None] + U * (ls[:, None] + lp.abs().nan_to_num(0.0, posinf=0.0)), "alternatives")
    if not gradient:
        return
    g = torch.Generator().manual_seed(seed)
    a, b = torch.randn(n, generator=g).cuda(), torch.randn(n, generator=g).cuda()
    leaf = x.detach().requires_grad_(True)
    lp, h = ops.token_log_probs(leaf, t, temperature=tau, top=top)[:2]
    assert torch.equal(lp.isnan(), out[0].isnan()) and torch.equal(lp.detach().nan_to_num(0), out[0].nan_to_num(0))
    for wa, wb in ((a, b), (a, None), (None, b)):
        got, = torch.autograd.grad([o for o, w in ((lp, wa), (h, wb)) if w is not None], leaf,
                                   [w for w in (wa, wb) if w is not None], retain_graph=True)
        assert got.dtype == x.dtype
        A = torch.zeros(n, device="cuda").double() if wa is None else wa.double()
        A = torch.where(given, A, 0.0)[:, None]
        B = torch.zeros_like(A) if wb is None else wb.double()[:, None]
        size = torch.where(p > 0, (log_p.abs() + want_h.abs()[:, None]), 0.0)
        want = -A * p - B * torch.where(p > 0, p * (log_p + want_h[:, None]), 0.0)
        hot = torch.zeros_like(want).scatter_(1, t.clamp(0, v - 1)[:, None].long(), A)
        want = (want + hot) / tau
        out_of = (A == 0) & (B == 0)
        want = torch.where(odd, torch.nan, torch.where((log_p.amax(1, keepdim=True) == -INF), 0.0, want))
        want = torch.where(out_of, 0.0, want)
        rel = (3 * y + 10) * U + es[:, None]
        bound = A.abs() * q * rel + B.abs() * q * (size.nan_to_num(0.0) * rel + eh[:, None] + es[:, None]
                                                   + (y + ls[:, None] + size.nan_to_num(0.0)) * 6 * U)
        bound = (bound + 4 * U * hot.abs()) / tau
        # exponentials below the smallest normal number may be 0
        bound = bound + (A.abs() + B.abs() * 300) / tau * 2.0 ** -125
        half, least = torch.finfo(x.dtype).eps / 2, torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps
        bound = bound + (want.abs().nan_to_num(0.0, posinf=0.0) + bound) * half * 1.001 + least
        close(got, want, bound, "gradient")


SIZES = [(1, 1, 1), (3, 7, 9), (2, 63, 5), (5, 64, 64), (4, 257, 1), (3, 1000, 16), (2, 4099, 256), (2, 20_011, 200),
         (70, 515, 30), (1100, 130, 12), (1030, 9001, 40), (1, 141_043, 20), (3, 100_003, 256)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,v,top", SIZES)
def test_sizes(ops, n, v, top, dtype):
    x, t = make(n, v, TYPES[dtype], seed=v + top)
    check(ops, x, t, tau=1.5, top=top)
    check(ops, x, t.int(), top=0, gradient=False)


@pytest.mark.parametrize("top", [1, 2, 8, 64, 255, 256])
@pytest.mark.parametrize("n,v", [(2, 300), (1100, 3000), (1030, 12_500), (2, 70_001)])
def test_tops(ops, n, v, top):
    for dtype in (torch.float32, torch.bfloat16):
        x, t = make(n, v, dtype, seed=top)
        check(ops, x, t, top=top, gradient=False)


def test_a_million_classes(ops):
    for n in (1, 40):
        x, t = make(n, 1_000_003, torch.bfloat16, seed=n)
        check(ops, x, t, top=100, gradient=n == 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 0), (5, 3), (2000, 1)])
def test_rows_that_start_anywhere(ops, pad, offset, dtype):
    for n, v in ((5, 1003), (3, 20_003), (1025, 2500)):
        x, t = make(n, v, TYPES[dtype], 1, pad, offset)
        check(ops, x, t, top=20, gradient=n < 1000)
    x, t = make(8, 700, TYPES[dtype], 2, pad, offset)
    check(ops, x[::2], t[1::2], top=3)


@pytest.mark.parametrize("n", [8, 1100])
@pytest.mark.parametrize("top", [1, 30, 256])
@pytest.mark.parametrize("v", [200, 5000, 30_000])
def test_orders_and_ties(ops, v, top, n):
    """Rows that rise, that fall, that are all equal, of few values, of alternating signs of 0, whose largest stand in one
    place, with all but a few masked."""
    x = torch.empty(8, v, device="cuda")
    i = torch.arange(v, device="cuda")
    x[0] = i * 1e-3
    x[1] = -i * 1e-3
    x[2] = 1.0
    x[3] = (i * 7919 % 5).float()
    x[4] = torch.where(i % 2 == 0, -0.0, 0.0)
    x[5] = -1.0
    x[5, v // 2:v // 2 + 150] = torch.arange(min(150, v - v // 2), device="cuda") % 40 + 1.0
    x[6] = -INF
    x[6, ::101] = 2.0
    x[7] = torch.finfo(torch.float32).min
    x[7, v - 3:] = torch.tensor([1.0, 2.0, 1.0], device="cuda")
    x = x.repeat(-(-n // 8), 1)[:n].contiguous()
    t = torch.arange(n, device="cuda") * 13 % v
    check(ops, x, t, top=top, gradient=False)
    half = x[:, :].bfloat16()
    check(ops, half, t, top=top, gradient=False)
    check(ops, x.flip(1).contiguous(), t, top=top, gradient=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1, 8, 100, 256])
def test_rows_that_flood_the_list_behind_a_cut(ops, top, dtype):
    """Whole rows by a workgroup each.  The second batch brings enough for the list to be cut, the next two more than
    there is room for, so that they are gone through again from what the cut had left."""
    n, batch = 1100, 1024 * (4 if dtype == "f32" else 8)
    v = 8 * batch + 77
    g = torch.Generator(device="cuda").manual_seed(top)
    x = torch.rand(n, v, generator=g, device="cuda")
    k = 3 * (top + max(8, top // 4))
    for i in range(0, n, 7):  # the same places in seven rows each
        at = batch + torch.randperm(batch, generator=g, device="cuda")[:k]
        x[i:i + 7, at] += 2.0
        at = 2 * batch + torch.randperm(2 * batch, generator=g, device="cuda")[:4000]
        x[i:i + 7, at] += 4.0
        at = 4 * batch + torch.randperm(4 * batch, generator=g, device="cuda")[:top // 2]
        x[i:i + 7, at] += 8.0
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    check(ops, x.to(TYPES[dtype]), t, top=top, gradient=False)


@pytest.mark.parametrize("v", [40, 3000, 60_003])
@pytest.mark.parametrize("times", [1, 120])
def test_masked_and_odd_logits(ops, v, times):
    low = torch.finfo(torch.float32).min
    x, _ = make(11, v, torch.float32, seed=v)
    t = torch.full((11,), 3, device="cuda")
    x[0, v // 2:] = -INF
    x[1, v // 2:] = low
    x[2] = low
    x[3] = -INF                 # nothing is left
    x[4, 3] = -INF              # the token is masked
    x[5, v // 3] = float("nan")
    x[6, v - 7] = INF
    x[7] = torch.finfo(torch.float32).max
    x[8, v - 1] = 1e30
    x[9] = -INF
    x[9, 3] = 1.0
    x[10] = -INF
    x[10, v - 2] = float("nan")
    t[10] = -1
    x, t = x.repeat(times, 1), t.repeat(times)
    check(ops, x, t, top=6)
    check(ops, x, t, tau=0.25, top=6)
    rows = [0, 3, 4, 5, 6, 9]
    check(ops, x[rows].bfloat16(), t[rows], top=50)


def test_tokens_outside(ops):
    x, _ = make(6, 500, torch.float32, seed=3)
    t = torch.tensor([-1, 500, 1 << 40, -(1 << 40), 499, 0], device="cuda")
    check(ops, x, t, top=4)
    check(ops, x, torch.tensor([-100, 500, 2 ** 31 - 1, -2 ** 31, 499, 0], device="cuda", dtype=torch.int32))


@pytest.mark.parametrize("tau", [1 / 1024, 0.05, 30.0, 1024.0])
def test_temperatures(ops, tau):
    x, t = make(5, 3001, torch.float32, seed=15)
    check(ops, x, t, tau=tau, top=10)


def test_rows_of_no_weight_are_not_looked_at(ops):
    x, t = make(4, 300, torch.bfloat16, seed=5)
    x[1] = float("nan")
    t[2] = -1
    leaf = x.requires_grad_(True)
    lp, h = ops.token_log_probs(leaf, t)
    g, = torch.autograd.grad((lp, h), leaf, (torch.tensor([1.0, 0.0, 1.0, 0.0], device="cuda"),
                                             torch.tensor([1.0, 0.0, 0.0, 0.0], device="cuda")))
    assert (g[1:] == 0).all() and (g[0] != 0).any()


def test_upstream_layouts(ops):
    x, t = make(8, 500, torch.float32, seed=8)
    leaf = x.requires_grad_(True)
    ones = torch.ones(8, device="cuda")
    want, = torch.autograd.grad(ops.token_log_probs(leaf, t)[0], leaf, ones)
    got, = torch.autograd.grad(ops.token_log_probs(leaf, t)[0].sum(), leaf)
    assert torch.equal(got, want)
    up = torch.randn(8, 2, device="cuda")
    got, = torch.autograd.grad(ops.token_log_probs(leaf, t), leaf, (up[:, 0], up[:, 1]))
    want, = torch.autograd.grad(ops.token_log_probs(leaf, t), leaf, (up[:, 0].contiguous(), up[:, 1].contiguous()))
    assert torch.equal(got, want)
    out = ops.token_log_probs(leaf, t, top=5)
    assert not out[2].requires_grad and not out[3].requires_grad and out[0].requires_grad
    # an expanded input: the gradients of its copies add up
    row = torch.randn(1, 500, device="cuda", requires_grad=True)
    (lp, h) = ops.token_log_probs(row.expand(8, 500), t)
    (lp.sum() + 0.5 * h.sum()).backward()
    each = row.detach().expand(8, 500).contiguous().requires_grad_(True)
    lp, h = ops.token_log_probs(each, t)
    g, = torch.autograd.grad(lp.sum() + 0.5 * h.sum(), each)
    assert torch.allclose(row.grad[0], g.sum(0), rtol=1e-5, atol=1e-6)
    with torch.no_grad():
        assert not ops.token_log_probs(leaf, t)[0].requires_grad


def test_gradient_against_differences(ops):
    """(f(S + h d) - f(S - h d)) / 2h of f = a log_prob + b entropy, directions of length 1, T = 2.  The third
    derivative along d of log sum exp(S / T) is a central moment, at most 0.0963 (2.83 / T) / T^2 < 0.04; that of the
    entropy has those up to the fourth times log p, at most 8 times as much: h = 1/8 is off by h^2 / 6 * 10 * 0.04 = 1e-3 at
    most; f below 10 is good to 2^-18: 10 * 2 * 2^-20 / 2h = 8e-5 more."""
    x, t = make(4, 60, torch.float32, seed=9, scale=1.0)
    a, b = torch.randn(4, device="cuda").clamp(-1, 1), torch.randn(4, device="cuda").clamp(-1, 1)
    leaf = x.clone().requires_grad_(True)
    grad, = torch.autograd.grad(ops.token_log_probs(leaf, t, temperature=2.0), leaf, (a, b))

    def f(x):
        lp, h = ops.token_log_probs(x, t, temperature=2.0)
        return a.double() * lp.double() + b.double() * h.double()

    h = 0.125
    for seed in range(5):
        d = torch.randn(4, 60, generator=torch.Generator().manual_seed(seed)).cuda()
        d /= d.norm(dim=1, keepdim=True)
        slope = (f(x + h * d) - f(x - h * d)) / (2 * h)
        assert ((grad.double() * d.double()).sum(1) - slope).abs().max() <= 1.1e-3


def test_the_binding_refuses(ops):
    x, t = make(4, 100, torch.float32, seed=10)
    for change in (dict(logits=x.double()), dict(logits=x[0]), dict(logits=x.t()), dict(logits=x[:, :0]), dict(logits=None),
                   dict(tokens=t.short()), dict(tokens=t[:3]), dict(tokens=t.cpu()), dict(tokens=t[:, None]),
                   dict(logits=torch.ones(4, 100, dtype=torch.complex64, device="cuda").conj().imag)):
        with pytest.raises(ValueError):
            ops.token_log_probs(**{"logits": x, "tokens": t, **change})
    from paper_1412_1576_amd.lda import LdaError
    for tau in (0.0, -1.0, float("nan"), 1e9):
        with pytest.raises(LdaError, match="temperature"):
            ops.token_log_probs(x, t, temperature=tau)
    with pytest.raises(LdaError, match="256"):
        ops.token_log_probs(x, t, top=257)
    with pytest.raises(LdaError, match="top"):
        ops.token_log_probs(x, t, top=-1)
    out = ops.token_log_probs(x[:0], t[:0], top=3)
    assert [o.shape for o in out] == [(0,), (0,), (0, 3), (0, 3)]
    none = x[:0].clone().requires_grad_(True)
    ops.token_log_probs(none, t[:0])[0].sum().backward()
    assert none.grad.shape == (0, 100)


def test_tangents_are_refused(ops):
    from torch.autograd import forward_ad
    x, t = make(4, 100, torch.float32, seed=10)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for on in (True, False):
            with torch.set_grad_enabled(on), pytest.raises(NotImplementedError):
                ops.token_log_probs(dual, t, top=3)


@pytest.mark.parametrize("stride", [1003, 1004, 1500])
@pytest.mark.parametrize("start", [0, 1, 7])
def test_gradient_rows_that_start_elsewhere(ops, stride, start):
    from paper_1412_1576_amd import lda
    n, v = 4, 1003
    x, t = make(n, v, torch.bfloat16, seed=3)
    leaf = x.clone().requires_grad_(True)
    lp, _ = ops.token_log_probs(leaf, t)
    want, = torch.autograd.grad(lp, leaf, torch.ones_like(lp))
    store = torch.full((n * stride + 16,), 5.0, dtype=torch.bfloat16, device="cuda")
    stats = ops._log_probs(x, t, 1.0, 0, True)[4]
    r = ops._log_prob_rows(x, t, 1.0, 0)
    one = torch.ones(1, device="cuda")
    L = lda.load_library()
    assert L.lda_log_probs_grad(r, stats.data_ptr(), one.data_ptr(), 0, None, 0, store.data_ptr() + 2 * start, stride) == 0
    torch.cuda.synchronize()
    rows = store[start:start + n * stride].view(n, stride)
    assert torch.equal(rows[:, :v], want)
    assert (rows[:, v:] == 5.0).all() and (store[:start] == 5.0).all() and (store[start + n * stride:] == 5.0).all()


def test_other_streams_and_two_calls_at_once(ops):
    big, small = make(4, 300_003, torch.bfloat16, 11), make(1100, 5003, torch.float32, 12)
    want = [ops.token_log_probs(*big, top=40), ops.token_log_probs(*small, top=40)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, data in zip(streams, (big, small)):
            with torch.cuda.stream(s):
                got.append(ops.token_log_probs(*data, top=40))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))


@pytest.mark.parametrize("n,v", [(3, 100_003), (1100, 515)])
def test_captured_and_replayed(ops, n, v):
    x, t = make(n, v, torch.bfloat16, seed=13)
    a = torch.rand(n, device="cuda")
    leaf = x.clone().requires_grad_(True)

    def step():
        out = ops.token_log_probs(leaf, t, top=17)
        return list(torch.autograd.grad(out[:2], leaf, (a, a))) + [o.detach() for o in out]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = step()
    for i in range(4):
        with torch.no_grad():
            leaf.copy_(make(n, v, torch.bfloat16, seed=20 + i)[0])
            a.uniform_()
            t.random_(0, v)
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, step()):
            assert torch.equal(g, w)
        torch.randn(1000, 1000, device="cuda").sum()


def test_rows_far_into_memory(ops):
    n, v = 15_500, 141_043    # 2.19 * 10^9 logits
    x = torch.zeros(n, v, dtype=torch.bfloat16, device="cuda")
    t = torch.randint(0, v, (n,), device="cuda")
    x[-3:] = torch.randn(3, v, device="cuda").to(x.dtype)
    far = ops.token_log_probs(x, t, top=20)
    near = ops.token_log_probs(x[-1100:].clone(), t[-1100:], top=20)
    # rows that start at the same place within 16 bytes: 14400 is a multiple of 8
    assert all(torch.equal(a[-1100:], b) for a, b in zip(far, near))
    leaf = x.requires_grad_(True)
    lp, h = ops.token_log_probs(leaf, t)
    got, = torch.autograd.grad((lp, h), leaf, (torch.ones_like(lp), torch.ones_like(h)))
    part = x.detach()[-1100:].clone().requires_grad_(True)
    lp, h = ops.token_log_probs(part, t[-1100:])
    want, = torch.autograd.grad((lp, h), part, (torch.ones_like(lp), torch.ones_like(h)))
    assert torch.equal(got[-1100:], want)


def test_more_rows_than_a_launch_has(ops):
    n, v = (1 << 20) + 5, 9
    x, t = torch.randn(n, v, device="cuda"), torch.randint(-1, v, (n,), device="cuda")
    check(ops, x, t, top=4)


def test_alternatives_teach(ops):
    """The alternatives are teacher rows of the distillation loss: all classes of a teacher, and a student of the same
    logits has no loss; of others the loss is the divergence."""
    x, t = make(6, 200, torch.float32, seed=21)
    _, _, ids, values = ops.token_log_probs(x, t, top=200)
    zero = torch.zeros(6, device="cuda")
    assert ops.distill_loss(x, ids, values, log_norm=zero).abs().max() <= 64 * U * 20
    other = make(6, 200, torch.float32, seed=22)[0]
    p, q = torch.log_softmax(x.double(), 1), torch.log_softmax(other.double(), 1)
    want = (p.exp() * (p - q)).sum(1)
    # masses are off by as much as log probabilities (below 30), each 30 roundings, and the terms are below 30
    assert (ops.distill_loss(other, ids, values, log_norm=zero) - want).abs().max() <= 30 * 64 * U
