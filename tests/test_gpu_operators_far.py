"""The operators on rows where positions pass 31 and 32 bits, with what is far against the same data near."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1412_1576_amd import operators
    return operators


def test_distillation_rows_far_into_memory(ops):
    n, v, k = 15_500, 141_043, 7    # 2.19 * 10^9 logits
    x = torch.zeros(n, v, dtype=torch.bfloat16, device="cuda")
    ids = torch.randint(0, v, (n, k), device="cuda")
    t = torch.randn(n, k, device="cuda")
    x[-3:] = torch.randn(3, v, device="cuda").to(x.dtype)
    loss, grad = ops.distill_loss_and_grad(x, ids, t)
    # the same kernel, and rows that start at the same place within 16 bytes (15500 - 204 is a multiple of 8): which
    # logits a thread sums is decided by that, and sums of other groups round otherwise
    near = ops.distill_loss_and_grad(x[-204:].clone(), ids[-204:], t[-204:])
    assert torch.equal(loss[-204:], near[0]) and torch.equal(grad[-204:], near[1])
    leaf = x.requires_grad_(True)
    loss = ops.distill_loss(leaf, ids, t)
    got, = torch.autograd.grad(loss, leaf, torch.ones_like(loss))
    part = x.detach()[-204:].clone().requires_grad_(True)
    loss_near = ops.distill_loss(part, ids[-204:], t[-204:])
    want, = torch.autograd.grad(loss_near, part, torch.ones_like(loss_near))
    assert torch.equal(loss.detach()[-204:], loss_near.detach()) and torch.equal(got[-204:], want)


def test_sequences_far_apart(ops):
    t, v, stride = 3, 30_011, (1 << 32) + 5
    g = torch.Generator().manual_seed(1)
    target = torch.softmax(torch.randn(2, t + 1, v, generator=g) * 2, 2).bfloat16().cuda()
    draft = torch.softmax(torch.randn(2, t, v, generator=g) * 2, 2).bfloat16().cuda()
    tokens = torch.multinomial(draft.float().cpu().view(2 * t, v), 1, generator=g).view(2, t).cuda()
    u, d = torch.rand(2, t, generator=g).cuda(), torch.rand(2, generator=g).cuda()
    store = torch.zeros(stride + (t + 1) * v, dtype=torch.bfloat16, device="cuda")
    far = store.as_strided((2, t + 1, v), (stride, v, 1))
    far.copy_(target)
    want = ops.verify_drafts(target, draft, tokens, u, d)
    got = ops.verify_drafts(far, draft, tokens, u, d)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_documents_far_into_an_assignment(ops):
    n = (1 << 31) + 300_000
    z = torch.full((n,), 5, dtype=torch.int32, device="cuda")
    z[-200_000:] = torch.randint(0, 40_000, (200_000,), dtype=torch.int32, device="cuda")
    ends = torch.tensor([0, 90, 4_000, 24_000, 200_000], device="cuda")
    near = ops.top_topics(z[-200_000:].clone(), ends, 40_000, 30, 0.1)
    far = ops.top_topics(z, ends + (n - 200_000), 40_000, 30, 0.1)
    for a, b in zip(far, near):
        assert torch.equal(a, b)
    # a document of 2^31 + 300000 tokens is cut at 2^31 - 1
    ids, logits, norm = ops.top_topics(z, torch.tensor([0, n], device="cuda"), 40_000, 2, 0.1)
    assert ids[0, 0] == 5 and abs(float(logits[0, 0].exp()) / (2 ** 31 - 1) - 1) < 1e-5


def test_more_rows_than_a_launch_has(ops):
    n, v = (1 << 20) + 5, 9
    x = torch.randn(n, v, device="cuda")
    ids, t = torch.randint(-1, v, (n, 3), device="cuda"), torch.randn(n, 3, device="cuda")
    loss, grad = ops.distill_loss_and_grad(x, ids, t)
    y = torch.log_softmax(x.double(), 1)
    p = torch.softmax(torch.where(ids >= 0, t.double(), -torch.inf), 1).nan_to_num(0.0)
    want = torch.where(p > 0, p * (p.log() - y.gather(1, ids.clamp(min=0))), 0.0).sum(1)
    assert (loss - want).abs().max() <= 64 * 2.0 ** -24 * 10   # logarithms below 10, some tens of roundings
    q = torch.zeros_like(y).scatter_add_(1, ids.clamp(min=0), p)
    want = (p.sum(1, keepdim=True) * y.exp() - q)
    assert (grad - want).abs().max() <= 64 * 2.0 ** -24


@pytest.mark.parametrize("v", [7, 5_000])
def test_more_sequences_than_a_launch_has(ops, v):
    n = (1 << 20) + 5
    p = torch.softmax(torch.randn(1, 1, v, device="cuda") * 2, 2)
    u = torch.rand(n, device="cuda")
    none = torch.zeros(n, 0, device="cuda")
    accepted, out = ops.verify_drafts(p.expand(n, 1, v), p[:, :0].expand(n, 0, v), none.long(), none, u)
    c = p[0, 0].double().cumsum(0)
    want = torch.searchsorted(c, u.double() * c[-1], right=True).clamp_(max=v - 1)
    assert (accepted == 0).all() and torch.equal(out[:, 0], want)
