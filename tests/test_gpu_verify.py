"""Verification of drafted tokens on the GPU against the rule in 64 bits, on the host.  Results are
whole numbers and have to be equal: a draw's place could be decided otherwise only where it lies within some 2^-45
of the border between two classes."""
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


def reference(target, draft, tokens, u, v, lengths=None):
    B, T = tokens.shape
    V = target.shape[2]
    accepted, out = np.zeros(B, np.int32), np.full((B, T + 1), -1, np.int64)
    with np.errstate(all="ignore"):
        for b in range(B):
            n = T if lengths is None else min(max(int(lengths[b]), 0), T)
            a = 0
            while a < n:
                x = int(tokens[b, a])
                if not 0 <= x < V or not float(u[b, a]) * draft[b, a, x] < target[b, a, x]:
                    break
                out[b, a] = x
                a += 1
            p = np.where(target[b, a] > 0, target[b, a], 0.0)
            mass = p
            if a < n:
                mass = target[b, a] - draft[b, a]
                mass = np.where(mass > 0, mass, 0.0)
                if not (mass > 0).any():
                    mass = p
            held = np.flatnonzero(mass > 0)
            if len(held):
                c = np.cumsum(mass[held])
                past = np.flatnonzero(c > float(v[b]) * c[-1])
                out[b, a] = held[past[0] if len(past) else -1]
            accepted[b] = a
    return accepted, out


def host(x):
    return x.double().cpu().numpy()


def check(ops, target, draft, tokens, u, v, lengths=None):
    want_a, want = reference(host(target), host(draft), tokens.cpu().numpy(), u.cpu().numpy(), v.cpu().numpy(),
                             None if lengths is None else lengths.cpu().numpy())
    accepted, out = ops.verify_drafts(target, draft, tokens, u, v, lengths=lengths)
    assert accepted.dtype == torch.int32 and out.dtype == tokens.dtype
    assert np.array_equal(accepted.cpu().numpy(), want_a)
    assert np.array_equal(out.cpu().numpy(), want)
    return want_a


def make(B, T, V, dtype, seed, sharp=3.0, near=0.7):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, T + 1, V, generator=g) * sharp
    target = torch.softmax(x, 2).to(dtype)
    draft = torch.softmax(x[:, :T] + near * torch.randn(B, T, V, generator=g), 2).to(dtype)
    tokens = torch.zeros(B, T, dtype=torch.int64)
    if T:
        tokens = torch.multinomial(draft.float().reshape(B * T, V), 1, generator=g).view(B, T)
    u = torch.rand(B, T, generator=g)
    v = torch.rand(B, generator=g)
    return [t.cuda() for t in (target, draft, tokens, u, v)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,T,V", [(1, 0, 1), (2, 1, 1), (3, 2, 7), (64, 4, 63), (33, 8, 1000), (5, 3, 4096),
                                   (7, 3, 4097), (40, 5, 8191), (2, 70, 300), (3, 1, 141_043)])
def test_sizes(ops, B, T, V, dtype):
    data = make(B, T, V, TYPES[dtype], seed=B + V)
    check(ops, *data)
    check(ops, *data[:2], data[2].int(), *data[3:])
    lengths = torch.randint(-1, T + 2, (B,), generator=torch.Generator().manual_seed(V), dtype=torch.int32)
    check(ops, *data, lengths=lengths.cuda())


def test_a_million_classes(ops):
    check(ops, *make(2, 2, 1_000_003, torch.bfloat16, seed=1, sharp=5.0))


def test_every_number_of_accepted_drafts_is_met(ops):
    met = check(ops, *make(400, 3, 50, torch.float32, seed=2))
    assert set(met.tolist()) == {0, 1, 2, 3}


def test_place_of_a_draw_on_the_borders(ops):
    """Masses that are powers of two: sums are exact, and a place that falls on a border goes to the
    class behind it."""
    V = 9000
    target = torch.zeros(1, 1, V)
    target[0, 0, [3, 4095, 4096, 8999]] = torch.tensor([0.25, 0.25, 0.125, 0.375])
    draws = torch.tensor([0.0, 0.249, 0.25, 0.49, 0.5, 0.624, 0.625, 0.99, 1.0, 1.5, -0.5, float("nan")])
    n = len(draws)
    target = target.expand(n, 1, V).cuda()
    none = torch.zeros(n, 0)
    got = ops.verify_drafts(target, torch.zeros(n, 0, V).cuda(), none.long().cuda(), none.cuda(), draws.cuda())[1]
    assert got[:, 0].tolist() == [3, 3, 4095, 4095, 4096, 4096, 8999, 8999, 8999, 8999, 3, 8999]


def test_odd_masses(ops):
    """Rows without mass, with NaN and infinity in them, target and draft alike, a rejected token of no
    probability, tokens outside the classes."""
    V, B = 5000, 10
    g = torch.Generator().manual_seed(3)
    target = torch.rand(B, 2, V, generator=g) / V
    draft = torch.rand(B, 1, V, generator=g) / V
    tokens = torch.randint(0, V, (B, 1), generator=g)
    u = torch.full((B, 1), 0.999999)
    target[0] = 0.0                                   # nothing to draw: -1
    target[1] = -1.0
    draft[2] = target[2, :1]                          # alike: accepted, as u < 1
    draft[3], u[3] = target[3, :1], 1.0               # alike and refused: drawn from the target
    target[4, 0, 17:4200] = float("nan")
    tokens[4] = 100
    target[5, :, 4500] = float("inf")
    draft[6] = 2 * target[6, :1]                      # the target has less everywhere
    tokens[7], tokens[8] = -1, V
    tokens[9] = 1 << 40
    v = torch.rand(B, generator=g)
    check(ops, *[t.cuda() for t in (target, draft, tokens, u, v)])


def test_rows_anywhere(ops):
    """Views of wider tensors, rows that start at any element, one draft and target for all sequences."""
    B, T, V = 6, 3, 5003
    target, draft, tokens, u, v = make(B, T, V, torch.bfloat16, seed=4)
    wide_t = torch.full((B, T + 2, V + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    wide_d = torch.full((B + 1, T + 1, V + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    wide_t[:, :T + 1, 5:V + 5] = target
    wide_d[1:, 1:, 1:V + 1] = draft
    wide_u = torch.rand(B, 2 * T, device="cuda")
    wide_u[:, 1:T + 1] = u
    check(ops, wide_t[:, :T + 1, 5:V + 5], wide_d[1:, 1:, 1:V + 1], tokens, wide_u[:, 1:T + 1], v)
    check(ops, target[:1].expand(B, -1, -1), draft[:1].expand(B, -1, -1), tokens, u, v)
    check(ops, target.transpose(0, 1)[:4].transpose(0, 1), draft, tokens, u, v)
    swapped = target.transpose(0, 1).contiguous().transpose(0, 1)
    check(ops, swapped, draft, tokens, u, v)


def test_output_rows_keep_what_lies_between(ops):
    import ctypes as C
    from paper_1412_1576_amd import lda
    B, T, V = 5, 2, 300
    target, draft, tokens, u, v = make(B, T, V, torch.float32, seed=5)
    want = ops.verify_drafts(target, draft, tokens, u, v)
    r = lda.lda_draft_rows()
    r.sequences, r.steps, r.classes = B, T, V
    r.target, r.target_sequence_stride, r.target_row_stride = target.data_ptr(), (T + 1) * V, V
    r.draft, r.draft_sequence_stride, r.draft_row_stride = draft.data_ptr(), T * V, V
    r.tokens, r.tokens_stride, r.tokens_type = tokens.data_ptr(), T, 1
    r.accept_u, r.accept_u_stride, r.draw_u = u.data_ptr(), T, v.data_ptr()
    r.hip_stream = torch.cuda.current_stream().cuda_stream
    L = lda.load_library()
    w = torch.empty(max(L.lda_verify_workspace(C.byref(r)), 1), dtype=torch.uint8, device="cuda")
    r.workspace, r.workspace_bytes = w.data_ptr(), w.numel()
    out = torch.full((B, 7), 99, dtype=torch.int64, device="cuda")
    accepted = torch.full((B + 2,), 99, dtype=torch.int32, device="cuda")
    assert L.lda_verify_drafts(C.byref(r), accepted.data_ptr(), out.data_ptr(), 7) == 0
    torch.cuda.synchronize()
    assert torch.equal(out[:, :3], want[1]) and (out[:, 3:] == 99).all()
    assert torch.equal(accepted[:B], want[0]) and (accepted[B:] == 99).all()


def test_draws_follow_the_target(ops):
    """One draft a sequence from q, kept or redrawn: the first token is distributed as p.  40000
    sequences over 8 classes; chi-square with 7 degrees of freedom is below 29.9 but for 1 in 10^4 --
    and the random numbers are fixed, so the outcome is."""
    n, V = 40_000, 8
    g = torch.Generator().manual_seed(6)
    p = torch.softmax(torch.randn(V, generator=g), 0)
    q = torch.softmax(torch.randn(V, generator=g), 0)
    tokens = torch.multinomial(q, n, replacement=True, generator=g).view(n, 1)
    target, draft = p.expand(n, 2, V).cuda(), q.expand(n, 1, V).cuda()
    out = ops.verify_drafts(target, draft, tokens.cuda(), torch.rand(n, 1, generator=g).cuda(),
                            torch.rand(n, generator=g).cuda())[1]
    seen = torch.bincount(out[:, 0].cpu(), minlength=V).double()
    want = p.double() / p.double().sum() * n
    assert ((seen - want) ** 2 / want).sum() < 29.9


def test_the_binding_refuses(ops):
    target, draft, tokens, u, v = make(2, 2, 30, torch.float32, seed=7)
    good = dict(target=target, draft=draft, tokens=tokens, accept_u=u, draw_u=v)
    for change in (dict(target=target.double()), dict(target=target[0]), dict(target=target.transpose(1, 2)),
                   dict(draft=draft.bfloat16()), dict(draft=draft[:, :1]), dict(tokens=tokens.float()),
                   dict(tokens=tokens[:1]), dict(accept_u=u.double()), dict(accept_u=u[:, :1]),
                   dict(draw_u=v[:1]), dict(draw_u=v.cpu()), dict(target=target[:, :0]),
                   dict(draw_u=v[:1].expand(2)), dict(lengths=tokens[:, 0]),
                   dict(lengths=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            ops.verify_drafts(**{**good, **change})
    accepted, out = ops.verify_drafts(target[:0], draft[:0], tokens[:0], u[:0], v[:0])
    assert accepted.shape == (0,) and out.shape == (0, 3)


@pytest.mark.parametrize("B,V", [(3, 50_003), (600, 300)])
def test_streams_and_graphs(ops, B, V):
    target, draft, tokens, u, v = make(B, 3, V, torch.float32, seed=8)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ops.verify_drafts(target, draft, tokens, u, v)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = ops.verify_drafts(target, draft, tokens, u, v)
        graphs.append((graph, got))
    for i in range(4):
        u.uniform_()
        v.uniform_()
        torch.cuda.synchronize()
        for (graph, _), stream in zip(graphs, (s, torch.cuda.current_stream())):
            with torch.cuda.stream(stream):   # both at once
                graph.replay()
        torch.cuda.synchronize()
        want = ops.verify_drafts(target, draft, tokens, u, v)
        for _, got in graphs:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check(ops, target, draft, tokens, u, v)


def test_streams_by_the_public_way(ops):
    for stream in (torch.cuda.default_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            device = torch.cuda.current_device()
            assert ops._stream_of(device) == ops._raw_stream(device) == stream.cuda_stream
