"""Root-mean-square norm on the GPU against the definition in 64 bits.  Tolerances count roundings (see
`bounds`)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1412_1576_amd import operators
    return operators


def half(t):
    return torch.finfo(t).eps / 2


def least(t):
    """Half a step of the numbers below the smallest normal one."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def sums(width):
    """Roundings of a sum over a row: a thread adds 16 numbers at most, or a 1024th of a wider row; 6 steps in a wave, 16
    waves."""
    return max(16, width / 1024 + 8) + 24


def make(n, width, dtype, seed, pad=0, offset=0, kind=None, scale=1.0):
    kind = kind or dtype
    g = torch.Generator().manual_seed(seed)
    store = torch.full((n * (width + pad) + offset + 8,), 777.0).to(kind)
    x = store[offset:offset + n * (width + pad)].view(n, width + pad)[:, :width]
    x.copy_((torch.randn(n, width, generator=g) * scale).to(kind))
    return store.cuda()[offset:offset + n * (width + pad)].view(n, width + pad)[:, :width]


def forward(h, w, eps):
    """(n, y, 1 / root) of the definition, float64 of what the tensors hold."""
    h = h.double()
    root = torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    n = torch.where(root == 0, 0.0, h / root)
    return n, n if w is None else n * w.double(), torch.where(root == 0, 0.0, 1 / root)


def rel(width):
    """Of n: half of what the sum of squares is off by, the mean's division, eps, root and quotient, two
    products."""
    return (sums(width) / 2 + 7) * U


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert torch.equal(got.isnan(), want.isnan()), what
    some = torch.isfinite(want)
    assert torch.equal(got[~some & ~want.isnan()], want[~some & ~want.isnan()]), what
    off = ((got - want).abs() - bound)[some]
    assert off.numel() == 0 or off.max() <= 0, (what, float(off.max()))


def check_sum(h, x, r):
    if r is None:
        return
    want = x.double() + r.double()
    close(h, want, want.abs() * (half(h.dtype) * 1.001 + (U if h.dtype != torch.float32 else 0)) + least(h.dtype), "sum")


def check(ops, x, w=None, r=None, eps=1e-6, gradient=True, seed=0):
    n, width = x.shape
    got = ops.rms_norm(x, w, residual=r, eps=eps)
    y, h = got if r is not None else (got, x)
    assert y.dtype == x.dtype and y.shape == x.shape and h.dtype == (x if r is None else r).dtype
    check_sum(h, x, r)
    eps32 = float(torch.tensor(eps, dtype=torch.float32))
    norm, want, inv = forward(h, w, eps32)
    close(y, want, want.abs() * (rel(width) + U + half(x.dtype) * 1.001) + least(x.dtype), "y")
    for dtype, most in ((torch.int8, 127.0), (torch.float8_e4m3fn, 448.0)):
        out = ops.rms_norm_8bit(x, w, residual=r, eps=eps, dtype=dtype)
        assert out[0].dtype == dtype and out[1].dtype == torch.float32
        if r is not None:
            assert torch.equal(out[2].nan_to_num(1), h.nan_to_num(1))
        top = want.abs().amax(1)
        top = torch.where(top < 2.0 ** -100, 0.0, top)  # such rows count as zeros
        odd = ~torch.isfinite(want).all(1)
        close(out[1], torch.where(odd, torch.nan, top / most), top.nan_to_num(0) / most * (rel(width) + 2 * U) + 1e-45, "scale")
        assert (out[0][odd].float() == 0).all()
        level = torch.where((top > 0)[:, None], want / (top / most)[:, None], 0.0)
        q = out[0].double()
        # y and the scale are both off, one more quotient and product
        slack = most * (2 * rel(width) + 6 * U)
        step = torch.full_like(level, 0.5) if dtype == torch.int8 else (level.abs() * 2.0 ** -4).clamp(min=2.0 ** -10)
        off = ((q - level).abs() - step - slack)[~odd]
        assert off.numel() == 0 or off.max() <= 0, dtype
        assert (q.abs() <= most).all()
    if not gradient:
        return
    g = torch.Generator().manual_seed(seed)
    gy = torch.randn(n, width, generator=g).to(x.dtype).cuda()
    gh = torch.randn(n, width, generator=g).to(h.dtype).cuda()
    leaves = [t.detach().requires_grad_(True) for t in (x, w, r) if t is not None]
    it = iter(leaves)
    xl, wl, rl = (next(it) if t is not None else None for t in (x, w, r))
    out = ops.rms_norm(xl, wl, residual=rl, eps=eps)
    grads = torch.autograd.grad(out, leaves, (gy, gh) if r is not None else gy)
    assert torch.equal((out[0] if r is not None else out).detach().nan_to_num(1), y.nan_to_num(1))
    gd = gy.double()
    u = gd if w is None else gd * w.double()
    along, size = (u * norm).mean(1, keepdim=True), (u * norm).abs().mean(1, keepdim=True)
    d = (u - norm * along) * inv
    # u is rounded once; the mean's terms are off as n is, and twice more, and its sum; then four roundings
    rn = rel(width)
    db = inv * (u.abs() * (rn + 5 * U) + norm.abs() * (size * (sums(width) * U + rn + 3 * U) + along.abs() * (2 * rn + 5 * U)))
    if r is not None:
        d = d + gh.double()
        db = db + (d.abs() + gh.double().abs()) * U
    by_leaf = dict(zip([name for name, t in (("x", x), ("w", w), ("r", r)) if t is not None], grads))
    close(by_leaf["x"], d, db + (d.abs() + db) * half(x.dtype) * 1.001 + least(x.dtype), "gradient of x")
    if r is not None:
        close(by_leaf["r"], d, db + (d.abs() + db) * half(h.dtype) * 1.001 + least(h.dtype), "gradient of the residual")
    if w is not None:
        gw = (gd * norm).sum(0)
        # rows of a group one by one (512 groups at least, or a row each), up to 2048 groups in 16 sums, these; a product
        gb = (gd * norm).abs().sum(0) * (rn + (n / 512 + min(n, 2048) / 16 + 19) * U)
        close(by_leaf["w"], gw, gb + (gw.abs() + gb) * half(w.dtype) * 1.001 + least(w.dtype), "gradient of the weight")


WIDTHS = [1, 7, 8, 9, 63, 64, 511, 512, 513, 1000, 2048, 2055, 4096, 5003, 8192, 10_001, 16_384, 16_385, 40_003]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(ops, width, dtype):
    t = TYPES[dtype]
    x = make(3, width, t, seed=width)
    check(ops, x)
    check(ops, x, make(1, width, t, seed=1)[0], make(3, width, t, seed=2))
    if dtype != "f32":
        check(ops, x, make(1, width, t, 1, kind=torch.float32)[0], make(3, width, t, 2, kind=torch.float32))
        check(ops, x, make(1, width, t, seed=1)[0], make(3, width, t, 2, kind=torch.float32))
        check(ops, x, make(1, width, t, 1, kind=torch.float32)[0])


@pytest.mark.parametrize("n,width", [(1, 4096), (511, 130), (513, 1000), (1700, 64), (2100, 2048), (600, 16_390)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows(ops, n, width, dtype):
    t = TYPES[dtype]
    check(ops, make(n, width, t, seed=n), make(1, width, t, seed=1)[0], make(n, width, t, seed=2))


@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 0), (24, 3)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_that_start_anywhere(ops, pad, offset, dtype):
    t = TYPES[dtype]
    for width in (500, 1003, 17_001):
        x, r = make(4, width, t, 1, pad, offset), make(4, width, t, 2, offset, pad)
        check(ops, x, make(1, width, t, 3, 0, offset)[0], r)
        check(ops, x[::2], None, r[1::2])


def test_sizes_of_numbers(ops):
    """Squares that leave 32 bits, rows of zeros, eps = 0."""
    x = make(9, 1000, torch.float32, seed=4)
    x *= torch.tensor([1e-38, 1e-30, 1e-20, 1e-10, 1.0, 1e10, 1e19, 1e25, 1e37], device="cuda")[:, None]
    w = make(1, 1000, torch.float32, seed=5)[0]
    check(ops, x, w, gradient=False)
    check(ops, x[1:], w, eps=0.0, gradient=False)
    check(ops, x[1:], w, eps=1e-30, gradient=False)
    check(ops, x[2:8], w, eps=0.0)
    check(ops, x[2:].bfloat16(), w.bfloat16(), eps=0.0, gradient=False)
    wide = make(3, 20_000, torch.float32, seed=4) * torch.tensor([1e-25, 1.0, 1e30], device="cuda")[:, None]
    check(ops, wide, eps=0.0, gradient=False)
    zero = torch.zeros(3, 700, device="cuda")
    zero[1] = 1.0
    for eps in (0.0, 1e-6):
        check(ops, zero, w[:700], eps=eps)
        q, scale = ops.rms_norm_8bit(zero, w[:700], eps=eps)
        assert scale[0] == 0 and (q[0] == 0).all() and scale[1] > 0


@pytest.mark.parametrize("n,width", [(2100, 300), (1100, 1500), (600, 4100), (520, 16_500)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_different_sizes(ops, n, width, dtype):
    """Orders of magnitude between neighbours, more rows than a gradient has workgroups: another row's root or scale would
    show."""
    size = 10.0 ** torch.randint(-6, 7, (n, 1), generator=torch.Generator().manual_seed(n), dtype=torch.float32).cuda()
    for kind in (None, torch.float32):
        x, r = make(n, width, TYPES[dtype], 1) * size.to(TYPES[dtype]), None
        if kind is not None:
            r = make(n, width, kind, 2) * size
        check(ops, x, make(1, width, TYPES[dtype], 3)[0], r, eps=0.0)


@pytest.mark.parametrize("width", [130, 3000, 20_000])
def test_numbers_that_are_none(ops, width):
    inf, nan = float("inf"), float("nan")
    x = make(4, width, torch.float32, seed=6)
    x[0, 5], x[1, width - 1], x[2, 0] = nan, inf, -inf
    check(ops, x, gradient=False)
    w = torch.ones(width, device="cuda")
    w[7] = nan
    check(ops, x, w, gradient=False)
    # a row of them leaves the others as they are
    clean = ops.rms_norm(x[3:])
    assert torch.equal(ops.rms_norm(x)[3:], clean)


def test_ties_go_to_even(ops):
    """Rows whose largest is 127 (448) of the scale: halves between levels are exact."""
    w = torch.arange(-127, 128, device="cuda").float() / 2.0
    w = torch.cat([w, torch.tensor([127.0], device="cuda")])
    x = torch.ones(1, 256, device="cuda")
    q, scale = ops.rms_norm_8bit(x, w, eps=0.0)
    assert float(scale[0]) == 1.0
    assert torch.equal(q[0].float(), torch.round(w))
    # from 16 on e4m3 has every second number
    v = torch.cat([torch.arange(16, 33, device="cuda").float(), torch.tensor([448.0], device="cuda")])
    q, scale = ops.rms_norm_8bit(torch.ones(1, 18, device="cuda"), v, eps=0.0, dtype=torch.float8_e4m3fn)
    assert float(scale[0]) == 1.0
    want = [16, 16, 18, 20, 20, 20, 22, 24, 24, 24, 26, 28, 28, 28, 30, 32, 32, 448]
    assert q[0].float().tolist() == [float(i) for i in want[:1] + want[1:]]


@pytest.mark.parametrize("value", [3.0, 0.7, 1e-4, 2.0 ** 70, 2.0 ** -70])
def test_ties_in_rows_of_any_root(ops, value):
    """All of a row's numbers are alike and the weights have the levels: the root leaves 32 bits, the ties remain."""
    w = torch.arange(-127, 128, device="cuda").float() / 2.0
    w = torch.cat([w, torch.tensor([127.0], device="cuda")])
    for x in (torch.full((3, 256), value, device="cuda"), torch.full((3, 256), value, device="cuda").bfloat16()):
        q, scale = ops.rms_norm_8bit(x, w, eps=1e-12)
        assert torch.equal(q.float(), torch.round(w).expand(3, 256))
    v = torch.cat([torch.arange(16, 33, device="cuda").float(), torch.tensor([448.0], device="cuda")])
    q, scale = ops.rms_norm_8bit(torch.full((2, 18), value, device="cuda"), v, eps=0.0, dtype=torch.float8_e4m3fn)
    want = [16, 16, 18, 20, 20, 20, 22, 24, 24, 24, 26, 28, 28, 28, 30, 32, 32, 448]
    assert q[0].float().tolist() == [float(i) for i in want]


@pytest.mark.parametrize("width", [100, 1000, 5000, 20_000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_levels_are_those_of_64_bits(ops, width, dtype):
    """A level is h w / max |h w| times the type's largest: 64 bits are off by some 2^-51 of it, so that numbers further from
    the middle of two levels than 2^-40 go to one side."""
    n = 400
    x, r = make(n, width, TYPES[dtype], 1), make(n, width, TYPES[dtype], 2, kind=torch.float32)
    for w in (None, make(1, width, TYPES[dtype], 3)[0]):
        for kind, most in ((torch.int8, 127.0), (torch.float8_e4m3fn, 448.0)):
            q, scale, h = ops.rms_norm_8bit(x, w, residual=r, dtype=kind)
            p = h.double() if w is None else h.double() * w.double()
            level = p / p.abs().amax(1, keepdim=True) * most
            if kind == torch.int8:
                step = torch.ones_like(level)
            else:
                step = torch.exp2(torch.floor(torch.log2(level.abs().clamp(min=2.0 ** -6))) - 3)
            places = level / step
            clear = (places - torch.floor(places) - 0.5).abs() > 2.0 ** -40
            assert torch.equal(q.double()[clear], (torch.round(places) * step)[clear])


def test_very_wide_rows_of_like_numbers(ops):
    """Each addition of a long sum in 32 bits would be rounded the same way.  A chunk's 8 numbers are added in 32 bits, the
    chunks in 64: 8 roundings of the squares, halved by the root, and seven more; the gradient's mean has 8 and six of its
    terms, then 8 roundings of numbers below 3."""
    width = 1 << 26
    x = torch.full((2, width), 1.1, device="cuda")
    x[1, ::3] = 0.3
    n, _, inv = forward(x, None, 1e-6)
    leaf = x.clone().requires_grad_(True)
    y = ops.rms_norm(leaf)
    close(y.detach(), n, n * (8 / 2 + 7 + 1) * U, "y")
    gy = torch.full_like(x, 0.7)
    got, = torch.autograd.grad(y, leaf, gy)
    want = (gy.double() - n * (gy.double() * n).mean(1, keepdim=True)) * inv
    close(got, want, 3 * (8 + 6 + 2 * 11 + 8) * U, "gradient")
    q, scale = ops.rms_norm_8bit(x)
    close(scale, n.amax(1) / 127, n.amax(1) / 127 * (8 / 2 + 7 + 3) * U, "scale")


def test_gradient_against_differences(ops):
    """(f(x + h d) - f(x - h d)) / 2h of f = sum(gy y) + sum(gh sum), rows of 60 with a mean square near 1, d of
    length 1.  n is smooth in x at the scale of the row's length, 7.7: a third derivative of gy y along d is at most
    30 |gy w| / 7.7^2 / root(60) of order 1, so that h = 1/16 is off by h^2 / 6 * 3 = 2e-3 at most; y is good to 40
    roundings, |f| < 60: 2 * 60 * 40 U / 2h = 2.3e-3 more."""
    x, r, w = (make(1, 60, torch.float32, seed=s) for s in (7, 8, 9))
    gy, gh = make(1, 60, torch.float32, seed=10), make(1, 60, torch.float32, seed=11)
    leaves = [t.clone().requires_grad_(True) for t in (x, w[0], r)]

    def f(x, w, r):
        y, h = ops.rms_norm(x, w, residual=r)
        return (y.double() * gy.double()).sum() + (h.double() * gh.double()).sum()

    grads = torch.autograd.grad(f(*leaves), leaves)
    h = 1 / 16
    for k in range(3):
        for seed in range(3):
            d = torch.randn(leaves[k].shape, generator=torch.Generator().manual_seed(seed)).cuda()
            d /= d.norm()
            up, down = ([t.detach() + (s * h * d if i == k else 0) for i, t in enumerate(leaves)] for s in (1, -1))
            slope = (f(*up) - f(*down)) / (2 * h)
            assert abs(float((grads[k].double() * d.double()).sum() - slope)) <= 4.3e-3


def test_which_gradients(ops):
    """Leaves that need none, outputs that are not used, broadcast inputs."""
    t = torch.bfloat16
    x, r, w = make(5, 300, t, 1), make(5, 300, t, 2, kind=torch.float32), make(1, 300, t, 3)[0]
    gy, gh = make(5, 300, t, 4), make(5, 300, t, 5, kind=torch.float32)

    def leaves():
        return [v.clone().requires_grad_(True) for v in (x, w, r)]

    xl, wl, rl = leaves()
    whole = torch.autograd.grad(ops.rms_norm(xl, wl, residual=rl), (xl, wl, rl), (gy, gh))
    for need in ((0,), (1,), (2,), (0, 1), (1, 2)):
        some = [v.clone().requires_grad_(i in need) for i, v in enumerate((x, w, r))]
        got = torch.autograd.grad(ops.rms_norm(some[0], some[1], residual=some[2]), [some[i] for i in need], (gy, gh))
        assert all(torch.equal(g, whole[i]) for g, i in zip(got, need))
    xl, wl, rl = leaves()
    got = torch.autograd.grad(ops.rms_norm(xl, wl, residual=rl)[0], (xl, wl, rl), gy)
    none = torch.autograd.grad(ops.rms_norm(xl, wl, residual=rl), (xl, wl, rl), (gy, torch.zeros_like(gh)))
    assert all(torch.equal(a, b) for a, b in zip(got, none))
    xl, wl, rl = leaves()
    ops.rms_norm(xl, wl, residual=rl)[1].backward(gh)
    assert torch.equal(rl.grad, gh) and torch.equal(xl.grad, gh.to(t)) and wl.grad is None
    # one type: the same gradient twice, in memory of its own for each leaf
    a, b = make(5, 300, t, 1).requires_grad_(True), make(5, 300, t, 2).requires_grad_(True)
    y, h = ops.rms_norm(a, residual=b)
    (y.sum() + h.sum()).backward()
    assert torch.equal(a.grad, b.grad)
    before = b.grad.clone()
    a.grad.zero_()
    assert torch.equal(b.grad, before)
    # upstream gradients of other layouts
    xl = x.clone().requires_grad_(True)
    one, = torch.autograd.grad(ops.rms_norm(xl).sum(), xl)
    same, = torch.autograd.grad(ops.rms_norm(xl), xl, torch.ones_like(x))
    assert torch.equal(one, same)
    across = make(300, 5, t, 6)
    got, = torch.autograd.grad(ops.rms_norm(xl), xl, across.t())
    want, = torch.autograd.grad(ops.rms_norm(xl), xl, across.t().contiguous())
    assert torch.equal(got, want)
    # one row for all: the gradients of its copies add up
    row = make(1, 300, torch.float32, 7).requires_grad_(True)
    gx, = torch.autograd.grad(ops.rms_norm(row.expand(5, 300)), row, gh)
    each = row.detach().expand(5, 300).contiguous().requires_grad_(True)
    ge, = torch.autograd.grad(ops.rms_norm(each), each, gh)
    assert torch.allclose(gx[0], ge.sum(0), rtol=1e-5, atol=1e-5)


def test_the_binding_refuses(ops):
    x, w = make(4, 100, torch.bfloat16, 1), make(1, 100, torch.bfloat16, 2)[0]
    for kw in (dict(x=x.double()), dict(x=x[0]), dict(x=x.t()), dict(x=x[:, :0]), dict(x=x.cpu()), dict(x=None),
               dict(weight=w.half()), dict(weight=w[:99]), dict(weight=w[:1].expand(100)), dict(residual=x.half()),
               dict(residual=x[:3]), dict(residual=x.double()),
               dict(residual=torch.ones(4, 100, dtype=torch.complex64, device="cuda").conj().imag)):
        kw = {"x": x, "weight": w, "residual": None, **kw}
        for call in (ops.rms_norm, ops.rms_norm_8bit):
            with pytest.raises(ValueError):
                call(**kw)
    with pytest.raises(ValueError):
        ops.rms_norm_8bit(x, dtype=torch.uint8)
    leaf = x.clone().requires_grad_(True)
    with pytest.raises(ValueError, match="gradient"):
        ops.rms_norm_8bit(leaf)
    with torch.no_grad():
        ops.rms_norm_8bit(leaf)
    from paper_1412_1576_amd.lda import LdaError
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(LdaError, match="eps"):
            ops.rms_norm(x, eps=eps)
    y, h = ops.rms_norm(x[:0], residual=x[:0])
    assert y.shape == h.shape == (0, 100)
    q, scale = ops.rms_norm_8bit(x[:0])
    assert q.shape == (0, 100) and scale.shape == (0,)
    none, wl = x[:0].clone().requires_grad_(True), w.clone().requires_grad_(True)
    ops.rms_norm(none, wl).sum().backward()
    assert none.grad.shape == (0, 100) and (wl.grad == 0).all()


def test_tangents_are_refused(ops):
    """Forward mode: a result without a tangent would stand for a derivative of zero."""
    from torch.autograd import forward_ad
    x, w, r = make(4, 100, torch.float32, 1), make(1, 100, torch.float32, 2)[0], make(4, 100, torch.float32, 3)
    with forward_ad.dual_level():
        for k in range(3):
            args = [x, w, r]
            args[k] = forward_ad.make_dual(args[k], torch.ones_like(args[k]))
            for on in (True, False):
                with torch.set_grad_enabled(on):
                    with pytest.raises(NotImplementedError):
                        ops.rms_norm(args[0], args[1], residual=args[2])
                    with pytest.raises(ValueError, match="gradient"):
                        ops.rms_norm_8bit(args[0], args[1], residual=args[2])
        assert torch.equal(ops.rms_norm(args[0], args[1], residual=args[2].detach())[0], ops.rms_norm(x, w, residual=r)[0])


def test_what_lies_between_rows_stays(ops):
    from paper_1412_1576_amd import lda
    x, stride = make(3, 1003, torch.bfloat16, 1), 1030
    want = ops.rms_norm(x)
    store = torch.full((3 * stride,), 5.0, dtype=torch.bfloat16, device="cuda")
    r = ops._norm_rows(x, x.stride(), None, None, None, 1e-6, 0)
    L = lda.load_library()
    assert L.lda_norm(r, store.data_ptr() + 2, stride, None, 0, None) == 0
    rows = store[1:1 + 2 * stride + 1003]
    assert torch.equal(rows.as_strided((3, 1003), (stride, 1), rows.storage_offset()), want)
    assert (store[0] == 5) and (store[1004:stride] == 5).all() and (store[1 + 2 * stride + 1003:] == 5).all()
    q, scale = ops.rms_norm_8bit(x)
    store = torch.full((3 * stride,), 77, dtype=torch.int8, device="cuda")
    other = torch.empty_like(scale)
    assert L.lda_norm_bytes(r, 0, store.data_ptr() + 1, stride, other.data_ptr(), None, 0) == 0
    rows = store[1:]
    assert torch.equal(rows.as_strided((3, 1003), (stride, 1), 1), q) and torch.equal(scale, other)
    assert (store[0] == 77) and (store[1004:stride] == 77).all()


def test_captured_and_replayed(ops):
    x, r, w = make(700, 1003, torch.bfloat16, 1), make(700, 1003, torch.bfloat16, 2, kind=torch.float32), \
        make(1, 1003, torch.bfloat16, 3)[0]
    gy = make(700, 1003, torch.bfloat16, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    leaves = [t.clone().requires_grad_(True) for t in (x, w, r)]

    def step():
        y, h = ops.rms_norm(leaves[0], leaves[1], residual=leaves[2])
        return [y.detach(), h.detach()] + list(torch.autograd.grad((y, h), leaves, (gy, h.detach()))) + \
            list(ops.rms_norm_8bit(leaves[0].detach(), leaves[1].detach()))

    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = step()
    for i in range(4):
        with torch.no_grad():
            leaves[0].copy_(make(700, 1003, torch.bfloat16, 10 + i))
            leaves[2].mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
        torch.randn(1000, 1000, device="cuda").sum()


def test_other_streams(ops):
    a, b = make(3000, 4096, torch.bfloat16, 1), make(500, 20_003, torch.float32, 2)
    want = [ops.rms_norm_8bit(a), ops.rms_norm_8bit(b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, x in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                got.append(ops.rms_norm_8bit(x))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


def test_rows_far_into_memory(ops):
    n, width = 140_000, 16_000      # 2.24 * 10^9 elements
    x = torch.zeros(n, width, dtype=torch.bfloat16, device="cuda")
    x[-600:] = make(600, width, torch.bfloat16, 1)
    part = x[-600:].clone()
    assert torch.equal(ops.rms_norm(x)[-600:], ops.rms_norm(part))
    q, scale = ops.rms_norm_8bit(x)
    qp, sp = ops.rms_norm_8bit(part)
    assert torch.equal(q[-600:], qp) and torch.equal(scale[-600:], sp) and (scale[:-600] == 0).all()
    del q
    leaf = x.requires_grad_(True)
    g, = torch.autograd.grad(ops.rms_norm(leaf), leaf, x.detach())
    near = part.clone().requires_grad_(True)
    gp, = torch.autograd.grad(ops.rms_norm(near), near, part)
    assert torch.equal(g[-600:], gp)


def test_the_widest_row(ops):
    """2^30 numbers, the most that a row may have: its norm, 8 bits and gradients, the weight's by more threads than a launch
    has.  The row is 1 but for a few larger numbers, here and there."""
    width = 1 << 30
    torch.cuda.empty_cache()
    x = torch.ones(1, width, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, (1 << 26) - 1, 1 << 26, (1 << 28) + 5, width // 2, width - 1], device="cuda")
    x[0, at] = torch.tensor([3.0, -2.0, 1.5, 100.0, 7.0, -0.5, 9.0], device="cuda").bfloat16()
    w = torch.ones(width, dtype=torch.bfloat16, device="cuda")
    w[at] = 2.0
    square = (width - 7 + 9 + 4 + 2.25 + 10_000 + 49 + 0.25 + 81) / width
    root = (square + 1e-6) ** 0.5
    leaf, wl = x.requires_grad_(True), w.requires_grad_(True)
    y = ops.rms_norm(leaf, wl)
    some = torch.cat([at, at[:-1] + 2])
    n = x.detach()[0, some].double() / root
    want = n * w.detach()[some].double()
    close(y.detach()[0, some], want, want.abs() * (12 * U + half(x.dtype) * 1.001), "y")
    gx, gw = torch.autograd.grad(y, (leaf, wl), torch.ones_like(y))
    close(gw[some], n, n.abs() * (13 * U + half(x.dtype) * 1.001), "gradient of the weight")
    # mean of w n over the row, the others are 1 / root each
    along = (width - 7 + 2 * (3.0 - 2.0 + 1.5 + 100.0 + 7.0 - 0.5 + 9.0)) / width / root
    u = w.detach()[some].double()
    d = (u - n * along) / root
    close(gx[0, some], d, (u + n.abs()) * 30 * U + d.abs() * half(x.dtype) * 1.001, "gradient of x")
    del y, gx, gw, leaf, wl
    q, scale = ops.rms_norm_8bit(x.detach(), w.detach())
    assert torch.equal(q[0, some].double(), torch.round(want / want.max() * 127))
    close(scale, want.max()[None] / 127, want.max() / 127 * 14 * U, "scale")
    del q, x, w
    torch.cuda.empty_cache()


def test_more_rows_than_a_launch_has(ops):
    n = (1 << 20) + 5
    x = torch.randn(n, 9, device="cuda")
    want = x.double() / torch.sqrt(x.double().square().mean(1, keepdim=True) + 1e-6)
    close(ops.rms_norm(x), want, want.abs() * (rel(9) + 2 * U), "y")
