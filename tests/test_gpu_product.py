"""Products of 8-bit integers on the GPU.  Sums are exact and the scaling is three roundings in a fixed order, so
that results are equal to the definition's, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1412_1576_amd import operators
    return operators


def integers(n, k, seed, pad=0, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    store = torch.full((n * (k + pad) + offset + 32,), 77, dtype=torch.int8, device="cuda")
    x = store[offset:offset + n * (k + pad)].view(n, k + pad)[:, :k]
    x.copy_(torch.randint(-128, 128, (n, k), generator=g, device="cuda", dtype=torch.int32).to(torch.int8))
    return x


def scales(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand(n, generator=g, device="cuda") * 0.01 + 1e-4


def definition(a, sa, b, sb, dtype):
    # (the sums are integers below 2^53: exact in 64-bit floating point, in any order)
    s = a.double() @ b.double().t().contiguous()
    assert s.abs().max() < 2 ** 31 if s.numel() else True
    # to 32 bits in one rounding, as an integer is
    return (s.float() * sa[:, None] * sb[None]).to(dtype)


def check(ops, a, b, dtype=torch.bfloat16, seed=1):
    sa, sb = scales(a.shape[0], seed), scales(b.shape[0], seed + 1)
    got = ops.int8_matmul(a, sa, b, sb, dtype=dtype)
    assert got.dtype == dtype
    want = definition(a, sa, b, sb, dtype)
    assert torch.equal(got, want), (got != want).sum()


ROWS = [1, 2, 15, 16, 17, 32, 33, 48, 49, 64, 65, 100, 128, 129, 300]


@pytest.mark.parametrize("k", [1, 15, 16, 63, 64, 65, 127, 128, 130, 256, 1000, 1024, 2064, 5120])
@pytest.mark.parametrize("n", [1, 17, 130])
def test_widths(ops, n, k):
    for m in (1, 20, 70):
        check(ops, integers(m, k, k), integers(n, k, k + 1))


@pytest.mark.parametrize("m", ROWS)
@pytest.mark.parametrize("n", [1, 16, 63, 129, 1000])
def test_rows_and_classes(ops, m, n):
    check(ops, integers(m, 256, m), integers(n, 256, n))
    check(ops, integers(m, 2051, m), integers(n, 2051, n))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 40_003, 512), (3, 17_000, 300), (20, 33_000, 272), (40, 33_001, 128), (64, 40_000, 144),
                                   (300, 70_003, 256), (1000, 20_000, 400), (2000, 30_011, 77), (257, 257, 4096),
                                   (700, 100, 16_384), (64, 48, 100_000)])
def test_shapes(ops, m, n, k, dtype):
    check(ops, integers(m, k, 1), integers(n, k, 2), TYPES[dtype])


@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (16, 0), (16, 16), (24, 8), (3, 5)])
@pytest.mark.parametrize("k", [96, 1040, 1111])
def test_rows_that_start_anywhere(ops, k, pad, offset):
    for m, n in ((5, 300), (200, 300)):
        check(ops, integers(m, k, 1, pad, offset), integers(n, k, 2))
        check(ops, integers(m, k, 1), integers(n, k, 2, pad, offset))
        check(ops, integers(2 * m, k, 1, pad, offset)[::2], integers(2 * n, k, 2, offset, pad)[1::2])
    # one row for all
    check(ops, integers(1, k, 1).expand(90, k), integers(300, k, 2))


@pytest.mark.parametrize("m", [65, 100, 128])
@pytest.mark.parametrize("k,pad,offset", [(77, 0, 0), (1000, 0, 0), (1008, 1, 0), (1008, 0, 1), (1008, 16, 0)])
def test_many_classes_of_rows_that_start_anywhere(ops, m, k, pad, offset):
    """As many classes as make tiles of 256 x 256, which read whole 16-byte pieces, and too few rows to be packed."""
    a, b = integers(m, k, 1), integers(200_003, k, 2, pad, offset)
    check(ops, a, b)
    if pad or offset:
        check(ops, integers(m, k, 1, pad, offset), integers(200_003, k, 2))


def test_rows_far_apart_and_many_classes(ops):
    """Rows so far apart that a place inside a tile leaves 32 bits."""
    store = torch.zeros(65, 1 << 24, dtype=torch.int8, device="cuda")
    a = store[:, 16:80]
    a.copy_(integers(65, 64, 1))
    check(ops, a, integers(200_003, 64, 2))


def test_the_largest_sums(ops):
    """Widths up to the largest with nothing but -128: the sum is 2^31 - 2^14."""
    for m in (1, 70):
        a = torch.full((m, 131_071), -128, dtype=torch.int8, device="cuda")
        b = torch.full((20, 131_071), -128, dtype=torch.int8, device="cuda")
        b[3] = 127
        check(ops, a, b, torch.float32)


def test_scales(ops):
    """Scales that are 0, infinite or no number, and results beyond 16 bits."""
    inf, nan = float("inf"), float("nan")
    for m in (4, 80):
        a, b = integers(m, 64, 1), integers(40, 64, 2)
        a[1] = 0
        sa, sb = scales(m, 3), scales(40, 4)
        sa[0], sa[2], sb[5], sb[6] = nan, 0.0, inf, 1e30
        for dtype in TYPES.values():
            got, want = ops.int8_matmul(a, sa, b, sb, dtype=dtype), definition(a, sa, b, sb, dtype)
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(1), want.nan_to_num(1))


def test_none(ops):
    a, b = integers(3, 0, 1), integers(5, 0, 2)
    assert torch.equal(ops.int8_matmul(a, scales(3, 1), b, scales(5, 2)), torch.zeros(3, 5, device="cuda").bfloat16())
    out = ops.int8_matmul(integers(3, 8, 1)[:0], scales(0, 1), integers(5, 8, 2), scales(5, 2))
    assert out.shape == (0, 5)


def test_the_binding_refuses(ops):
    a, b, sa, sb = integers(4, 64, 1), integers(8, 64, 2), scales(4, 3), scales(8, 4)
    for kw in (dict(a=a.short()), dict(a=a[0]), dict(a=a.t()), dict(a=a.cpu()), dict(b=b.byte()), dict(b=b[:, :32]),
               dict(b=b[:0]), dict(a_scale=sa[:3]), dict(a_scale=sa.double()), dict(a_scale=sa[:1].expand(4)), dict(b_scale=sb[:7]),
               dict(b_scale=sb[:, None]), dict(dtype=torch.float64), dict(b_scale=sb.clone().requires_grad_(True)),
               dict(a_scale=torch.ones(4, dtype=torch.complex64, device="cuda").conj().imag)):
        with pytest.raises(ValueError):
            ops.int8_matmul(**{"a": a, "a_scale": sa, "b": b, "b_scale": sb, **kw})
    from paper_1412_1576_amd.lda import LdaError
    wide = torch.zeros(1, 131_072, dtype=torch.int8, device="cuda")
    with pytest.raises(LdaError, match="131071"):
        ops.int8_matmul(wide, sa[:1], wide, sb[:1])


def test_tangents_are_refused(ops):
    from torch.autograd import forward_ad
    a, b, sa, sb = integers(4, 64, 1), integers(8, 64, 2), scales(4, 3), scales(8, 4)
    with forward_ad.dual_level():
        for scale in ((forward_ad.make_dual(sa, sa), sb), (sa, forward_ad.make_dual(sb, sb))):
            with pytest.raises(ValueError, match="gradient"), torch.no_grad():
                ops.int8_matmul(a, scale[0], b, scale[1])


@pytest.mark.parametrize("m,n", [(3, 100), (100, 300), (600, 70_000)])
def test_what_lies_between_rows_stays(ops, m, n):
    from paper_1412_1576_amd import lda
    a, b, sa, sb = integers(m, 64, 1), integers(n, 64, 2), scales(m, 3), scales(n, 4)
    want = ops.int8_matmul(a, sa, b, sb)
    stride = n + 7
    store = torch.full((m * stride + 16,), 5.0, dtype=torch.bfloat16, device="cuda")
    r = lda.lda_product_rows(m, n, 64, a.data_ptr(), 64, sa.data_ptr(), b.data_ptr(), 64, sb.data_ptr(), 2, 0, None, 0,
                             torch.cuda.current_stream().cuda_stream)
    assert lda.load_library().lda_product(r, store.data_ptr() + 2, stride) == 0
    torch.cuda.synchronize()
    rows = store[1:1 + m * stride].view(m, stride)
    assert torch.equal(rows[:, :n], want) and (rows[:, n:] == 5).all() and store[0] == 5 and (store[1 + m * stride:] == 5).all()


def test_captured_and_replayed(ops):
    cases = [(integers(m, k, 1), scales(m, 2), integers(n, k, 3), scales(n, 4))
             for m, n, k in ((5, 64, 8192), (130, 200, 4096), (300, 60_000, 256))]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for c in cases:
            ops.int8_matmul(*c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = [ops.int8_matmul(*c) for c in cases]
    for i in range(4):
        for c in cases:
            c[0].copy_(integers(*c[0].shape, 10 + i))
            c[1].mul_(1.1)
        graph.replay()
        torch.cuda.synchronize()
        for g, c in zip(got, cases):
            assert torch.equal(g, ops.int8_matmul(*c))
        torch.randn(1000, 1000, device="cuda").sum()


def test_other_streams_and_two_calls_at_once(ops):
    cases = [(integers(m, k, 1), scales(m, 2), integers(n, k, 3), scales(n, 4))
             for m, n, k in ((20, 48, 65_536), (130, 200, 16_384))]
    want = [ops.int8_matmul(*c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                got.append(ops.int8_matmul(*c))
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_far_into_memory(ops):
    """Weights and results whose positions pass 31 and 32 bits."""
    b = integers(1_100_000, 4000, 1)     # 4.4 * 10^9 bytes
    sb = scales(1_100_000, 2)
    for m in (3, 100):
        a, sa = integers(m, 4000, 3), scales(m, 4)
        got = ops.int8_matmul(a, sa, b, sb)
        want = definition(a, sa, b[-3000:], sb[-3000:], torch.bfloat16)
        assert torch.equal(got[:, -3000:], want)
    del b
    a, b = integers(40_000, 64, 5), integers(70_000, 64, 6)   # 2.8 * 10^9 results
    sa, sb = scales(40_000, 7), scales(70_000, 8)
    got = ops.int8_matmul(a, sa, b, sb)
    want = definition(a[-300:], sa[-300:], b, sb, torch.bfloat16)
    assert torch.equal(got[-300:], want)


def test_as_many_classes_as_there_may_be(ops):
    """2^31 - 1 classes: the first, those about the launches' and the middle's borders, and the last."""
    n = 2 ** 31 - 1
    torch.cuda.empty_cache()
    b, sb = integers(n, 1, 1), scales(n, 2)
    for m in (1, 9):    # by the few-rows kernel, by tiles
        a, sa = integers(m, 1, 3), scales(m, 4)
        got = ops.int8_matmul(a, sa, b, sb)
        for at in (0, 2 ** 22 * 64 - 1000, 2 ** 30 - 1000, n - 2000):
            some = slice(at, at + 2000)
            assert torch.equal(got[:, some], definition(a, sa, b[some], sb[some], torch.bfloat16))
        del got
    del b, sb
    torch.cuda.empty_cache()


def test_a_head(ops):
    """Norm to 8 bits, product, log probabilities: hidden rows to what is read off their logits, against the same from
    the numbers that the 8 bits stand for."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x, r = (torch.randn(70, 512, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.rand(512, generator=g, device="cuda") + 0.5
    b = integers(3001, 512, 9)
    sb = torch.full((3001,), 1e-3, device="cuda")
    q, scale, h = ops.rms_norm_8bit(x, w, residual=r)
    logits = ops.int8_matmul(q, scale, b, sb, dtype=torch.float32)
    tokens = torch.randint(0, 3001, (70,), generator=g, device="cuda")
    lp, entropy, ids, values = ops.token_log_probs(logits, tokens, top=5)
    exact = (q.double() * scale.double()[:, None]) @ (b.double() * 1e-3).t().contiguous()
    # logits are three roundings of 2^-24 off, and 1e-3 one more: 4 of numbers below 30; a log probability is a difference
    # of two of them, rounded some 40 times more on its way
    p = torch.log_softmax(exact, 1)
    assert exact.abs().max() < 30
    assert (lp - p.gather(1, tokens[:, None])[:, 0]).abs().max() <= 30 * (2 * 4 + 60) * 2.0 ** -24
    assert torch.equal(ids, logits.topk(5, dim=1)[1].int())
    assert torch.equal(h, (x.float() + r.float()).bfloat16())
    student = torch.randn(70, 3001, generator=g, device="cuda", requires_grad=True)
    ops.distill_loss(student, ids, values, log_norm=torch.zeros(70, device="cuda")).mean().backward()
    assert torch.isfinite(student.grad).all()
    # the answers to a batch: a class drawn from each row of probabilities
    probs = torch.softmax(logits, 1)[:, None]
    none = torch.zeros(70, 0, device="cuda")
    accepted, drawn = ops.verify_drafts(probs, probs[:, :0], none.long(), none, torch.rand(70, generator=g, device="cuda"))
    assert (accepted == 0).all() and ((drawn >= 0) & (drawn < 3001)).all()
