"""Refusals of the operators on rows that need no GPU: the library's own checks of sizes, types,
pointers and alignment, and the binding's checks of tensors."""
import ctypes as C
import os

import pytest
import torch

from paper_1412_1576_amd import lda


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lda.LIB_PATH):
        from paper_1412_1576_amd import build
        build.build_library()
    return lda.load_library()


def message(lib):
    return lib.lda_last_error(None).decode()


def distill(**kw):
    r = lda.lda_distill_rows()
    r.rows, r.classes, r.slots = 4, 1000, 8
    r.logits, r.logits_stride, r.ids, r.ids_stride = 1 << 20, 1000, 1 << 20, 8
    r.teacher, r.teacher_stride, r.temperature = 1 << 20, 8, 1.0
    for k, v in kw.items():
        setattr(r, k, v)
    return r


@pytest.mark.parametrize("field,value,code", [
    ("rows", -1, lda.LDA_ERR_ARG), ("classes", 0, lda.LDA_ERR_ARG), ("slots", -1, lda.LDA_ERR_ARG),
    ("slots", 1025, lda.LDA_ERR_UNSUPPORTED), ("logits_type", 3, lda.LDA_ERR_ARG),
    ("teacher_type", -1, lda.LDA_ERR_ARG), ("ids_type", 2, lda.LDA_ERR_ARG),
    ("temperature", 0.0, lda.LDA_ERR_ARG), ("temperature", -1.0, lda.LDA_ERR_ARG),
    ("temperature", float("nan"), lda.LDA_ERR_ARG), ("temperature", float("inf"), lda.LDA_ERR_ARG),
    ("temperature", 2.0 ** -11, lda.LDA_ERR_ARG), ("logits", None, lda.LDA_ERR_ARG),
    ("ids", None, lda.LDA_ERR_ARG), ("teacher", None, lda.LDA_ERR_ARG),
    ("logits", (1 << 20) + 2, lda.LDA_ERR_ARG), ("ids", (1 << 20) + 2, lda.LDA_ERR_ARG),
    ("log_norm", (1 << 20) + 1, lda.LDA_ERR_ARG), ("weight", (1 << 20) + 1, lda.LDA_ERR_ARG)])
def test_distill_refuses(lib, field, value, code):
    r = distill(**{field: value})
    out = 1 << 21
    for call, args in (("lda_distill_workspace", ()), ("lda_distill_loss", (out, out)),
                       ("lda_distill_grad", (out, out, 1000)), ("lda_distill_step", (out, out, 1000))):
        assert getattr(lib, call)(C.byref(r), *args) == code, call
        assert call in message(lib)


def test_distill_refuses_outputs_and_workspaces(lib):
    r, out = distill(), 1 << 21
    assert lib.lda_distill_loss(C.byref(r), None, out) == lda.LDA_ERR_ARG
    assert lib.lda_distill_loss(C.byref(r), out + 1, out) == lda.LDA_ERR_ARG
    assert lib.lda_distill_grad(C.byref(r), None, out, 1000) == lda.LDA_ERR_ARG
    assert lib.lda_distill_grad(C.byref(r), out, None, 1000) == lda.LDA_ERR_ARG
    assert lib.lda_distill_grad(C.byref(r), out, out, 999) == lda.LDA_ERR_ARG and "overlap" in message(lib)
    assert lib.lda_distill_step(C.byref(r), out, out + 2, 1000) == lda.LDA_ERR_ARG
    assert lib.lda_distill_workspace(None) == lda.LDA_ERR_ARG
    r.reserved[2] = 1
    assert lib.lda_distill_step(C.byref(r), out, out, 1000) == lda.LDA_ERR_ARG
    big = distill(rows=1, classes=1_000_000, logits_stride=1_000_000)
    need = lib.lda_distill_workspace(C.byref(big))
    assert need > 0
    for pointer, nbytes in ((None, need), (1 << 21, need - 1), ((1 << 21) + 8, need)):
        big.workspace, big.workspace_bytes = pointer, nbytes
        assert lib.lda_distill_loss(C.byref(big), out, out) == lda.LDA_ERR_ARG
        assert "workspace" in message(lib)


def test_no_rows_are_no_work(lib):
    r = distill(rows=0, logits=None, ids=None, teacher=None)
    assert lib.lda_distill_workspace(C.byref(r)) == 0
    assert lib.lda_distill_loss(C.byref(r), None, None) == lda.LDA_OK
    assert lib.lda_distill_step(C.byref(r), None, None, 0) == lda.LDA_OK
    assert lib.lda_distill_grad(C.byref(r), None, None, 0) == lda.LDA_OK
    d = draft(sequences=0, target=None)
    assert lib.lda_verify_workspace(C.byref(d)) == 0
    assert lib.lda_verify_drafts(C.byref(d), None, None, 0) == lda.LDA_OK
    assert lib.lda_top_topics(C.byref(topics(rows=0)), None, None, None) == lda.LDA_OK


def draft(**kw):
    r = lda.lda_draft_rows()
    r.sequences, r.steps, r.classes = 2, 3, 100_000
    for name in ("target", "draft", "tokens", "accept_u", "draw_u", "workspace"):
        setattr(r, name, 1 << 20)
    r.workspace_bytes = 1 << 20
    for k, v in kw.items():
        setattr(r, k, v)
    return r


@pytest.mark.parametrize("field,value,code", [
    ("sequences", -1, lda.LDA_ERR_ARG), ("steps", -1, lda.LDA_ERR_ARG), ("classes", 0, lda.LDA_ERR_ARG),
    ("steps", 4097, lda.LDA_ERR_UNSUPPORTED), ("probs_type", 3, lda.LDA_ERR_ARG),
    ("tokens_type", 2, lda.LDA_ERR_ARG), ("target", None, lda.LDA_ERR_ARG),
    ("draft", None, lda.LDA_ERR_ARG), ("tokens", None, lda.LDA_ERR_ARG),
    ("accept_u", None, lda.LDA_ERR_ARG), ("draw_u", None, lda.LDA_ERR_ARG),
    ("target", (1 << 20) + 2, lda.LDA_ERR_ARG), ("lengths", (1 << 20) + 2, lda.LDA_ERR_ARG),
    ("workspace", None, lda.LDA_ERR_ARG), ("workspace_bytes", 0, lda.LDA_ERR_ARG),
    ("workspace", (1 << 20) + 8, lda.LDA_ERR_ARG)])
def test_verify_refuses(lib, field, value, code):
    r = draft(**{field: value})
    assert lib.lda_verify_drafts(C.byref(r), 1 << 21, 1 << 21, 4) == code
    assert "lda_verify_drafts" in message(lib)


def test_verify_refuses_outputs(lib):
    r, out = draft(), 1 << 21
    assert lib.lda_verify_drafts(C.byref(r), None, out, 4) == lda.LDA_ERR_ARG
    assert lib.lda_verify_drafts(C.byref(r), out, None, 4) == lda.LDA_ERR_ARG
    assert lib.lda_verify_drafts(C.byref(r), out, out + 2, 4) == lda.LDA_ERR_ARG
    assert lib.lda_verify_drafts(C.byref(r), out, out, 3) == lda.LDA_ERR_ARG and "overlap" in message(lib)
    assert lib.lda_verify_drafts(None, out, out, 4) == lda.LDA_ERR_ARG
    r.reserved[0] = 1
    assert lib.lda_verify_drafts(C.byref(r), out, out, 4) == lda.LDA_ERR_ARG


def topics(**kw):
    r = lda.lda_topic_rows()
    r.rows, r.documents, r.K, r.tokens, r.slots, r.alpha = 2, 2, 10, 5, 4, 0.1
    r.offsets = r.z = 1 << 20
    for k, v in kw.items():
        setattr(r, k, v)
    return r


@pytest.mark.parametrize("field,value,code", [
    ("rows", -1, lda.LDA_ERR_ARG), ("rows", 3, lda.LDA_ERR_ARG), ("documents", -1, lda.LDA_ERR_ARG),
    ("tokens", -1, lda.LDA_ERR_ARG), ("K", 0, lda.LDA_ERR_ARG), ("K", 2 ** 20 - 1, lda.LDA_ERR_UNSUPPORTED),
    ("slots", 0, lda.LDA_ERR_ARG), ("slots", 1025, lda.LDA_ERR_UNSUPPORTED), ("alpha", 0.0, lda.LDA_ERR_ARG),
    ("alpha", float("nan"), lda.LDA_ERR_ARG), ("alpha", float("inf"), lda.LDA_ERR_ARG),
    ("offsets_type", 2, lda.LDA_ERR_ARG), ("offsets", None, lda.LDA_ERR_ARG), ("z", None, lda.LDA_ERR_ARG),
    ("z", (1 << 20) + 1, lda.LDA_ERR_ARG), ("docs", (1 << 20) + 2, lda.LDA_ERR_ARG),
    ("reserved_word", 1, lda.LDA_ERR_ARG), ("workspace", 8, lda.LDA_ERR_ARG),
    ("workspace_bytes", -1, lda.LDA_ERR_ARG)])
def test_top_topics_refuses(lib, field, value, code):
    r = topics(**{field: value})
    assert lib.lda_top_topics(C.byref(r), 1 << 21, 1 << 21, 1 << 21) == code
    assert "lda_top_topics" in message(lib)
    assert lib.lda_topics_workspace(C.byref(r)) == code


def test_topics_refuse_outputs_and_contexts(lib):
    out = 1 << 21
    assert lib.lda_top_topics(C.byref(topics()), None, out, out) == lda.LDA_ERR_ARG
    assert lib.lda_top_topics(C.byref(topics()), out, None, out) == lda.LDA_ERR_ARG
    assert lib.lda_top_topics(C.byref(topics()), out, out + 1, out) == lda.LDA_ERR_ARG
    assert lib.lda_top_topics(None, out, out, out) == lda.LDA_ERR_ARG
    assert lib.lda_doc_topics(None, 1, None, 4, out, out, out) == lda.LDA_ERR_ARG


def test_struct_layouts():
    # (rows; classes, slots; 6 of logits, ids, teacher; log_norm; weight, its stride; 4 words; workspace,
    # bytes, stream; reserved) and so on, all fields at their natural alignment
    assert C.sizeof(lda.lda_distill_rows) == 8 + 8 + 6 * 8 + 8 + 16 + 16 + 24 + 16
    assert C.sizeof(lda.lda_draft_rows) == 8 + 8 + 3 * 8 + 3 * 8 + 2 * 8 + 8 + 2 * 8 + 8 + 8 + 24 + 16
    assert C.sizeof(lda.lda_topic_rows) == 3 * 8 + 8 + 8 + 2 * 8 + 8 + 8 + 2 * 8 + 8 + 16


def test_the_binding_refuses_host_tensors():
    from paper_1412_1576_amd import operators
    x = torch.zeros(2, 5)
    i = torch.zeros(2, 3, dtype=torch.int64)
    with pytest.raises(ValueError, match="on the GPU"):
        operators.distill_loss(x, i, torch.zeros(2, 3))
    with pytest.raises(ValueError, match="on the GPU"):
        operators.distill_loss_and_grad(x, i, torch.zeros(2, 3))
    with pytest.raises(ValueError, match="on the GPU"):
        operators.verify_drafts(torch.zeros(1, 2, 5), torch.zeros(1, 1, 5), i[:1, :1], x[:1, :1], x[0, :1])
    with pytest.raises(ValueError, match="on the GPU"):
        operators.top_topics(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int64), 4, 2, 0.1)
    with pytest.raises(ValueError, match="on the GPU"):
        operators.distill_loss(None, i, x)


def test_the_import_needs_nothing_private_of_torch(monkeypatch):
    import importlib
    from paper_1412_1576_amd import operators
    with monkeypatch.context() as without:
        without.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
        importlib.reload(operators)
        assert operators._raw_stream is operators._stream_of
    importlib.reload(operators)
