"""Top topics of documents on the GPU against counting on the host; from tensors and from a sampler.
Ids are equal; a logit is the logarithm in 64 bits rounded once (half a step, 2^-24), of a value that the
host's differs from by 2^-50 at most."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1412_1576_amd import operators
    return operators


def reference(z, offsets, K, slots, alpha, docs):
    n = len(docs)
    ids, logits, norm = np.full((n, slots), -1), np.full((n, slots), -np.inf), np.zeros(n)
    for i, d in enumerate(docs):
        part = z[offsets[d]:offsets[d + 1]] if 0 <= d < len(offsets) - 1 else z[:0]
        part = part[(part >= 0) & (part < K)]
        topic, count = np.unique(part, return_counts=True)
        order = np.lexsort((topic, -count))[:slots]
        ids[i, :len(order)] = topic[order]
        logits[i, :len(order)] = np.log(count[order] + alpha)
        norm[i] = np.log(len(part) + K * alpha)
    return ids, logits, norm


def same(got, want):
    ids, logits, norm = [x.cpu().numpy() for x in got]
    assert np.array_equal(ids, want[0])
    for g, w in ((logits, want[1]), (norm, want[2])):
        some = np.isfinite(w)
        assert np.array_equal(g[~some], w[~some].astype(np.float32))
        assert (np.abs(g[some] - w[some]) <= np.abs(w[some]) * 2.0 ** -24 * 1.001 + 1e-15).all()


def check(ops, z, lengths, K, slots, alpha=0.1, docs=None, dtype=np.int64):
    offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(dtype)
    z = np.ascontiguousarray(z[:offsets[-1]], np.int32)
    on = None if docs is None else torch.tensor(np.asarray(docs, np.int32)).cuda()
    got = ops.top_topics(torch.from_numpy(z).cuda(), torch.from_numpy(offsets).cuda(), K, slots, alpha, docs=on)
    same(got, reference(z, offsets, K, slots, alpha, range(len(lengths)) if docs is None else docs))
    return got


def some_z(rng, n, K, flat=0.5):
    few = rng.integers(0, K, 9)
    return np.where(rng.random(n) < flat, rng.integers(0, K, n), few[rng.integers(0, 9, n)])


@pytest.mark.parametrize("slots", [1, 8, 100, 1024])
@pytest.mark.parametrize("K", [1, 10, 1000, 12_289, 1_000_000])
def test_sizes(ops, K, slots):
    rng = np.random.default_rng(K + slots)
    lengths = np.concatenate([[0, 1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1023, 1024, 1025],
                              rng.integers(0, 300, 40), [2047, 2048, 2049, 4095, 4096, 4097, 5000, 0]])
    check(ops, some_z(rng, lengths.sum(), K), lengths, K, slots)


@pytest.mark.parametrize("K", [3, 5000, 100_000, 2 ** 20 - 2])
def test_long_documents(ops, K):
    rng = np.random.default_rng(K)
    lengths = [30_000, 8191, 8192, 8193, 0, 16_384, 200_000, 12_288, 12_289, 65_537]
    z = some_z(rng, sum(lengths), K)
    check(ops, z, lengths, K, 64, dtype=np.int32)
    check(ops, z, lengths, K, 1000)


@pytest.mark.parametrize("length", [50, 64, 100, 500, 3000, 40_000])
def test_ties_and_extremes(ops, length):
    """Every topic once, every topic twice, one topic alone: ties go to the lower topic."""
    K = 100_000
    each = np.arange(length)[::-1] * (K // length)
    twice = np.repeat(np.arange(length // 2), 2)[::-1]
    z = np.concatenate([each, twice, np.full(length, K - 1), np.full(length, 0)])
    lengths = [length, len(twice), length, length]
    check(ops, z, lengths, K, 7)
    check(ops, z, lengths, K, 300)


def test_topics_outside_and_documents_outside(ops):
    rng = np.random.default_rng(1)
    lengths = rng.integers(0, 200, 50)
    lengths[7] = 9000
    z = some_z(rng, lengths.sum(), 40)
    z[::3] = rng.choice([-1, 40, 41, 2 ** 31 - 1, -2 ** 31, 2 ** 20 - 1], len(z[::3]))
    check(ops, z, lengths, 40, 16)
    check(ops, z, lengths, 40, 16, docs=[3, 7, 7, -1, 50, 49, 0, 2 ** 31 - 1, 3])
    check(ops, z, lengths, 40, 16, docs=[])


def test_bad_offsets_are_clamped(ops):
    z = torch.arange(10, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([-5, 3, 2, 8, 1 << 40, 4], device="cuda")
    ids, logits, norm = ops.top_topics(z, offsets, 10, 4, 1.0)
    assert ids.tolist() == [[0, 1, 2, -1], [-1] * 4, [2, 3, 4, 5], [8, 9, -1, -1], [-1] * 4]
    assert norm.exp().round().int().tolist() == [13, 10, 16, 12, 10]


def test_an_empty_assignment(ops):
    z = torch.zeros(0, dtype=torch.int32, device="cuda")
    ids, logits, norm = ops.top_topics(z, torch.zeros(4, dtype=torch.int64, device="cuda"), 5, 2, 0.5)
    assert (ids == -1).all() and torch.isneginf(logits).all() and ids.shape == (3, 2)
    assert torch.allclose(norm, torch.full((3,), 2.5, device="cuda").log(), rtol=2.0 ** -23)
    assert ops.top_topics(z, torch.zeros(1, dtype=torch.int64, device="cuda"), 5, 2, 0.5)[0].shape == (0, 2)


def test_the_binding_refuses(ops):
    from paper_1412_1576_amd.lda import LdaError
    z = torch.zeros(6, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 3, 6], device="cuda")
    for args in ((z.long(), off, 4, 2, 0.1), (z, off.float(), 4, 2, 0.1), (z, off[:0], 4, 2, 0.1),
                 (z[::2], off, 4, 2, 0.1), (z, off, 1 << 40, 2, 0.1), (z.view(2, 3), off, 4, 2, 0.1)):
        with pytest.raises(ValueError):
            ops.top_topics(*args)
    for args in ((z, off, 0, 2, 0.1), (z, off, 4, 0, 0.1), (z, off, 4, 2000, 0.1), (z, off, 4, 2, 0.0),
                 (z, off, 2 ** 20, 2, 0.1), (z, off, 4, -3, 0.1)):
        with pytest.raises(LdaError):
            ops.top_topics(*args)
    with pytest.raises(ValueError):
        ops.top_topics(z, off, 4, 2, 0.1, docs=off)


def test_captured_and_replayed(ops):
    K, D = 500, 300
    rng = np.random.default_rng(2)
    lengths = rng.integers(0, 150, D)
    lengths[5] = 10_000
    offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)])).cuda()
    z = torch.randint(0, K, (int(lengths.sum()),), dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ops.top_topics(z, offsets, K, 16, 0.1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = ops.top_topics(z, offsets, K, 16, 0.1)
    for _ in range(3):
        z.random_(0, K)
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, ops.top_topics(z, offsets, K, 16, 0.1)):
            assert torch.equal(g, w)


@pytest.mark.parametrize("own_stream", [False, True])
def test_of_a_sampler(ops, own_stream):
    """lda_doc_topics against the sampler's own assignment, in every state, on its stream."""
    from paper_1412_1576_amd import corpus, lda
    cfg = corpus.scaled(corpus.CONFIGS["c1"], D=200)
    doff, words = corpus.make_corpus(cfg)
    stream = torch.cuda.Stream() if own_stream else None
    m = lda.Lda(doff, words, cfg.V, cfg.K, cfg.alpha, cfg.beta, seed=3,
                stream=stream.cuda_stream if own_stream else None)
    for it in range(3):
        same(m.doc_topics(20), reference(m.get_z(), doff, cfg.K, 20, cfg.alpha, range(200)))
        m.build_alias()
        m.sweep(2)
        got = m.doc_topics(20, torch.tensor([5, 199, 0, 5, -1, 200], dtype=torch.int32, device="cuda"))
        same(got, reference(m.get_z(), doff, cfg.K, 20, cfg.alpha, [5, 199, 0, 5, -1, 200]))
        m.rebuild_counts()
    row = m.get_ndk_row(7)
    ids, logits, _ = m.doc_topics(cfg.K)
    assert ids[7, :int((row > 0).sum())].sort()[0].tolist() == np.flatnonzero(row).tolist()
    with pytest.raises(lda.LdaError, match="1024"):
        m.doc_topics(1025)
    with pytest.raises(lda.LdaError):
        m.doc_topics(0)
    with pytest.raises(ValueError):
        m.doc_topics(4, torch.zeros(2, device="cuda"))
    m.close()


def test_of_a_streamed_sampler(ops):
    from paper_1412_1576_amd import corpus, lda
    cfg = corpus.scaled(corpus.CONFIGS["c1"], D=200)
    doff, words = corpus.make_corpus(cfg)
    m = lda.Lda(doff, words, cfg.V, cfg.K, cfg.alpha, cfg.beta, stream_block_tokens=5000)
    with pytest.raises(lda.LdaError, match="streamed"):
        m.doc_topics(4)
    m.close()


def test_together(ops):
    """The operators as they are used: a sampler's documents are the teacher, a student of one linear
    layer over the documents' words learns their topics, proposes topics for new tokens, and its proposals
    are verified against the sampler's own theta."""
    from paper_1412_1576_amd import corpus, lda
    cfg = corpus.scaled(corpus.CONFIGS["c1"], D=400)
    doff, words = corpus.make_corpus(cfg)
    m = lda.Lda(doff, words, cfg.V, cfg.K, cfg.alpha, cfg.beta, seed=1)
    for _ in range(5):
        m.build_alias()
        m.sweep(2)
        m.rebuild_counts()
    ids, logits, log_norm = m.doc_topics(cfg.K)
    # theta is what the rows stand for: all of the document's topics have a slot
    theta = torch.zeros(cfg.D, cfg.K, dtype=torch.float64)
    for d in range(0, cfg.D, 57):
        row = m.get_ndk_row(d)
        theta[d] = torch.from_numpy((row + cfg.alpha) / (row.sum() + cfg.K * cfg.alpha))
    bag = torch.zeros(cfg.D, cfg.V, device="cuda")
    doc = torch.from_numpy(np.repeat(np.arange(cfg.D), np.diff(doff))).cuda()
    bag.index_put_((doc, torch.from_numpy(words).long().cuda()), torch.ones(len(words), device="cuda"),
                   accumulate=True)
    student = torch.nn.Linear(cfg.V, cfg.K, device="cuda")
    out = student(bag)
    loss = ops.distill_loss(out, ids, logits, log_norm=log_norm)
    loss.mean().backward()
    q = torch.softmax(out.detach().double(), 1).cpu()
    for d in range(0, cfg.D, 57):
        # logits and norm carry 2^-24 of up to 5 each, theta then 1e-6; the loss that of log theta too
        want = (theta[d] * (theta[d].log() - q[d].log())).sum()
        assert abs(float(loss.detach()[d]) - float(want)) <= 1e-5 * max(1.0, float(want))
    step = ops.distill_loss_and_grad(out.detach(), ids, logits, log_norm=log_norm,
                                     weight=torch.full((cfg.D,), 1.0 / cfg.D, device="cuda"))
    assert torch.equal(step[0], loss.detach())
    want = step[1].t() @ bag
    assert torch.allclose(student.weight.grad, want, rtol=1e-4, atol=1e-6)
    # four topics proposed for each document from the student, against theta
    docs = torch.arange(0, cfg.D, 57)
    p = theta[docs][:, None].expand(-1, 5, -1).float().cuda()
    draft = q[docs][:, None].expand(-1, 4, -1).float().cuda()
    tokens = torch.multinomial(q[docs], 4, replacement=True).cuda()
    accepted, got = ops.verify_drafts(p, draft, tokens, torch.rand(len(docs), 4, device="cuda"),
                                      torch.rand(len(docs), device="cuda"))
    for i, a in enumerate(accepted.tolist()):
        assert torch.equal(got[i, :a], tokens[i, :a]) and 0 <= got[i, a] < cfg.K and (got[i, a + 1:] == -1).all()
    m.close()


@pytest.mark.parametrize("K", [40_000, 100_000, 400_000, 2 ** 20 - 2])
def test_any_workspace_gives_the_same(ops, K):
    """None, room for one of the long documents, room for all: rows are equal, what lies around them is as it
    was; the documents' topics are few (tables, joined ranges) or many (counters)."""
    import ctypes as C
    from paper_1412_1576_amd import lda
    rng = np.random.default_rng(K)
    lengths = [70_000, 20_000, 3, 65_536, 65_535, 150_000, 16_384, 16_383, 0, 30_000, 90_000]
    z = some_z(rng, sum(lengths), K, flat=0.3)
    z[:70_000] = rng.integers(0, 300, 70_000)     # a few topics, many tokens
    z[70_000:90_000] = rng.integers(0, K, 20_000)
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    zt, ot = torch.from_numpy(z.astype(np.int32)).cuda(), torch.from_numpy(offsets).cuda()
    slots, n = 100, len(lengths)
    want = reference(z, offsets, K, slots, 0.1, range(n))
    L = lda.load_library()
    r = lda.lda_topic_rows(n, None, n, ot.data_ptr(), 1, K, zt.data_ptr(), zt.numel(), slots, 0, 0.1, None, 0,
                           torch.cuda.current_stream().cuda_stream)
    need = L.lda_topics_workspace(r)
    assert need > 0
    one = 16 + 8 + -(-K // 31_744) * (8 + 8 * slots)
    for nbytes in (0, 15, one, 2 * one, need):
        w = torch.full((max(nbytes, 1) + 64,), 255, dtype=torch.uint8, device="cuda")
        r.workspace, r.workspace_bytes = w.data_ptr() if nbytes else None, nbytes
        out = [torch.full((n + 1, slots), -77, dtype=torch.int32, device="cuda"),
               torch.full((n + 1, slots), -77.0, device="cuda"), torch.full((n + 1,), -77.0, device="cuda")]
        assert L.lda_top_topics(r, *[x.data_ptr() for x in out]) == 0
        torch.cuda.synchronize()
        same([x[:n] for x in out], want)
        assert all((x[n:] == -77).all() for x in out) and (w[nbytes:] == 255).all()


def test_a_sampler_captured(ops):
    """On the sampler's own stream the call is captured and replayed; on another one it is refused."""
    from paper_1412_1576_amd import corpus, lda
    cfg = corpus.scaled(corpus.CONFIGS["c1"], D=150)
    doff, words = corpus.make_corpus(cfg)
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    m = lda.Lda(doff, words, cfg.V, cfg.K, cfg.alpha, cfg.beta, seed=4, stream=stream.cuda_stream)
    docs = torch.tensor([3, 0, 149], dtype=torch.int32, device="cuda")
    with torch.cuda.stream(stream):
        m.doc_topics(10, docs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = m.doc_topics(10, docs)
    for picked in ([3, 0, 149], [7, 7, 8], [100, -1, 150]):
        docs.copy_(torch.tensor(picked, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        same(got, reference(m.get_z(), doff, cfg.K, 10, cfg.alpha, picked))
    with pytest.raises(ValueError, match="captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=other):
            m.doc_topics(10, docs)
    torch.cuda.synchronize()
    same(m.doc_topics(10, docs), reference(m.get_z(), doff, cfg.K, 10, cfg.alpha, [100, -1, 150]))
    m.close()


def test_a_sampler_captured_and_swept(ops):
    """A captured call replayed after sweeps and new assignments reads the assignment that there is then, whichever of
    the sampler's two buffers has it."""
    from paper_1412_1576_amd import corpus, lda
    cfg = corpus.scaled(corpus.CONFIGS["c1"], D=150)
    doff, words = corpus.make_corpus(cfg)
    stream = torch.cuda.Stream()
    m = lda.Lda(doff, words, cfg.V, cfg.K, cfg.alpha, cfg.beta, seed=4, stream=stream.cuda_stream)
    with torch.cuda.stream(stream):
        m.doc_topics(10)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = m.doc_topics(10)

    def replayed():
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        same(got, reference(m.get_z(), doff, cfg.K, 10, cfg.alpha, range(cfg.D)))

    replayed()
    for _ in range(3):
        m.build_alias()
        m.sweep(2)
        replayed()
        m.rebuild_counts()
    rng = np.random.default_rng(3)
    for _ in range(2):
        m.set_z(rng.integers(0, cfg.K, len(words)).astype(np.int32), m.sweep_index)
        replayed()
    m.close()


def test_a_sweep_captured_with_its_topics(ops):
    """An iteration and its topics in one graph, with sweeps by the host between the replays; and the topics in a
    graph of their own."""
    from paper_1412_1576_amd import corpus, lda
    cfg = corpus.scaled(corpus.CONFIGS["c1"], D=150)
    doff, words = corpus.make_corpus(cfg)
    stream = torch.cuda.Stream()

    def iterate(m):
        m.build_alias()
        m.sweep(2)
        m.rebuild_counts()

    m = lda.Lda(doff, words, cfg.V, cfg.K, cfg.alpha, cfg.beta, seed=5, stream=stream.cuda_stream)
    other = lda.Lda(doff, words, cfg.V, cfg.K, cfg.alpha, cfg.beta, seed=5, stream=stream.cuda_stream)
    with torch.cuda.stream(stream):
        for _ in range(2):
            iterate(m)
        m.doc_topics(10)
    torch.cuda.synchronize()
    before, index = m.get_z(), m.sweep_index
    m.set_z(before, index)  # a sweep captured after another one goes on from what that one has drawn ahead
    m.rebuild_counts()
    graph, alone = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        iterate(m)
        got = m.doc_topics(10)
    with torch.cuda.graph(alone, stream=stream):
        after = m.doc_topics(10)

    def one_sweep_from(z):
        other.set_z(z, index)
        other.rebuild_counts()
        iterate(other)
        return other.get_z()

    # the graph sweeps from one of the two buffers into the other; the host's sweeps take the assignment back into
    # the first, from the second after the capture and from the first itself later
    for sweeps in (1, 2, 2):
        with torch.cuda.stream(stream):
            graph.replay()
            alone.replay()
        torch.cuda.synchronize()
        z = one_sweep_from(before)
        for rows in (got, after):
            same(rows, reference(z, doff, cfg.K, 10, cfg.alpha, range(cfg.D)))
        m.rebuild_counts()
        for _ in range(sweeps):
            iterate(m)
            before = m.get_z()
            with torch.cuda.stream(stream):
                alone.replay()
            torch.cuda.synchronize()
            same(after, reference(before, doff, cfg.K, 10, cfg.alpha, range(cfg.D)))
    m.close()
    other.close()


def test_a_sampler_on_another_device(ops, monkeypatch):
    """The call goes to the sampler's device, whichever is the current one, and leaves that as it was."""
    from paper_1412_1576_amd import corpus, lda
    cfg = corpus.scaled(corpus.CONFIGS["c1"], D=50)
    doff, words = corpus.make_corpus(cfg)
    m = lda.Lda(doff, words, cfg.V, cfg.K, cfg.alpha, cfg.beta, seed=6)
    want = reference(m.get_z(), doff, cfg.K, 10, cfg.alpha, range(cfg.D))
    device = torch.cuda.current_device()
    docs = torch.arange(cfg.D, dtype=torch.int32, device="cuda")
    made = []
    with monkeypatch.context() as other:  # the program's device is the next one
        other.setattr(torch.cuda, "current_device", lambda: device + 1)
        other.setattr(torch.cuda, "set_device", made.append)
        got = [m.doc_topics(10), m.doc_topics(10, docs)]
    assert made == [device, device + 1] * 2
    for rows in got:
        assert all(x.get_device() == device for x in rows)
        same(rows, want)
    if torch.cuda.device_count() > 1:
        with torch.cuda.device((device + 1) % torch.cuda.device_count()):
            same(m.doc_topics(10), want)
            ids = torch.empty(cfg.D, 10, dtype=torch.int32, device=device)
            rc = lda.load_library().lda_doc_topics(m._h, cfg.D, None, 10, ids.data_ptr(), ids.data_ptr(), None)
            assert rc == lda.LDA_ERR_ARG
    m.close()


@pytest.mark.parametrize("K", [1000, 1024, 1025, 5000])
@pytest.mark.parametrize("rows", [7_000, 14_000])
def test_waves_with_several_documents(ops, rows, K):
    """More documents than the GPU has waves (6144), then more than two each (from there on the logarithms come from
    tables): a wave gets empty, short and middle ones, some with too many topics for it and some too long for it, in
    every order, and what it leaves goes to workgroups with several rows each."""
    rng = np.random.default_rng(rows + K)
    kind = rng.choice(5, rows, p=[0.1, 0.5, 0.2, 0.17, 0.03])
    lengths = np.select([kind == 0, kind == 1, kind == 2, kind == 3],
                        [0, rng.integers(1, 91, rows), rng.integers(300, 700, rows), rng.integers(700, 1_500, rows)],
                        rng.integers(4_096, 4_300, rows))
    after = {(a, b) for a, b in zip(kind[:-6144], kind[6144:])}
    assert len(after) >= (25 if rows > 12_288 else 20)  # each kind after each in the same wave
    owner = np.repeat(np.arange(rows), lengths)
    z = np.where((kind[owner] == 3) | (rng.random(len(owner)) < 0.4), rng.integers(0, K, len(owner)),
                 (rng.integers(0, 9, len(owner)) * 7919 + owner * 31) % K)
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    many = [d for d in np.flatnonzero(kind == 3)[:200] if len(np.unique(z[offsets[d]:offsets[d + 1]])) > 512]
    assert len(many) > 20
    check(ops, z, lengths, K, 24)
    check(ops, z, lengths, K, 24, docs=rng.integers(-1, rows + 1, rows), dtype=np.int32)


@pytest.mark.parametrize("length,K,alpha", [(300, 100, 0.01), (20_000, 1000, 0.05), (440_000, 100, 0.01), (2_000_000, 1000, 0.01)])
def test_the_floor_that_the_rows_stand_for(ops, length, K, alpha):
    """What a document's rows leave for the classes without a slot, from the gradient at one of them: T (M q - r) with
    equal logits, q = 1 / K.  Each mass is off by half a step of its logit and of the norm, 2^-24 of their size, the rest
    by as much of 1; the gradient by some roundings of q."""
    rng = np.random.default_rng(length)
    few = rng.permutation(K)[:K * 6 // 10]
    z = torch.from_numpy(few[rng.integers(0, len(few), length)].astype(np.int32)).cuda()
    ids, logits, norm = ops.top_topics(z, torch.tensor([0, length], device="cuda"), K, min(K, 1024), alpha)
    _, grad = ops.distill_loss_and_grad(torch.zeros(1, K, device="cuda"), ids, logits, log_norm=norm)
    named = np.unique(z.cpu().numpy())
    others = np.setdiff1d(np.arange(K), named)
    r = 1.0 / K - grad[0, others].double().cpu().numpy()
    size = float(norm[0])
    off = 2.0 ** -24 * (np.log(length) + size + 2) + len(others) * 8 * 2.0 ** -24 / K
    assert np.abs(r * len(others) - len(others) * alpha / (length + K * alpha)).max() <= off
    got = torch.exp(logits[0].double() - norm[0].double()).cpu().numpy()[:len(named)]
    counts = np.bincount(z.cpu().numpy(), minlength=K)[ids[0].cpu().numpy()[:len(named)]]
    want = (counts + alpha) / (length + K * alpha)
    assert (np.abs(got - want) <= want * 2.0 ** -23 * size).all()
