"""The library's operators on rows, on torch tensors of the GPU (lda_mi355x.h has their definitions).

  top_topics, Lda.doc_topics   documents' most frequent topics as the top logits of a teacher
  distill_loss                 distillation from a teacher's top logits, with autograd
  distill_loss_and_grad        the same and its gradient in one call, for weights known beforehand
  verify_drafts                drafted tokens accepted or redrawn from given random numbers

Work goes to torch's current stream of the tensors' device; outputs and workspaces come from
torch's allocator; no call waits for the GPU.  Wrong shapes, types or devices raise ValueError,
refusals of the library LdaError.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import lda
from .lda import LDA_OK, LdaError

_FLOATS = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_INDEXES = {torch.int32: 0, torch.int64: 1}
_INT32 = 2 ** 31 - 1


def _tensor(x, name, dims, types, device=None, spread=False):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError("%s must be a tensor on the GPU" % name)
    if x.dtype not in types:
        raise ValueError("%s must be one of %s, not %s" % (name, ", ".join(map(str, types)), x.dtype))
    if x.dim() != dims:
        raise ValueError("%s must have %d dimensions, not %d" % (name, dims, x.dim()))
    if device is not None and x.device != device:
        raise ValueError("%s is on %s, not on %s" % (name, x.device, device))
    if not spread and x.stride(-1) != 1 and x.size(-1) > 1:
        raise ValueError("%s: elements of a row must be adjacent (call .contiguous())" % name)
    if x.size(-1) > _INT32 and dims > 1:
        raise ValueError("%s: a row has at most 2^31 - 1 elements" % name)


def _int32(x, name):
    x = int(x)
    if not -_INT32 <= x <= _INT32:
        raise ValueError("%s does not fit 32 bits" % name)
    return x


def _shape(x, name, shape):
    if tuple(x.shape) != tuple(shape):
        raise ValueError("%s has shape %s, not %s" % (name, tuple(x.shape), tuple(shape)))


def _check(rc):
    if rc < LDA_OK:
        raise LdaError(rc, (lda.load_library().lda_last_error(None) or b"").decode())
    return rc


class _On:
    """The tensors' device as the current one, for the length of a call."""

    def __init__(self, device):
        self.device = device

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.device.index:
            torch.cuda.set_device(self.device)

    def __exit__(self, *exc):
        if self.before != self.device.index:
            torch.cuda.set_device(self.before)


def _workspace(r, nbytes, device):
    """Room for the call; the caching allocator keeps it from work of other streams."""
    if nbytes == 0:
        return None
    w = torch.empty(nbytes, dtype=torch.uint8, device=device)
    r.workspace, r.workspace_bytes = w.data_ptr(), nbytes
    return w


def _distill_rows(logits, ids, teacher, temperature, log_norm, weight=None, weight_stride=0):
    device = logits.device
    r = lda.lda_distill_rows()
    r.rows, r.classes = logits.shape
    r.slots = ids.shape[1]
    r.logits, r.logits_stride = logits.data_ptr(), logits.stride(0)
    r.ids, r.ids_stride = ids.data_ptr(), ids.stride(0)
    r.teacher, r.teacher_stride = teacher.data_ptr(), teacher.stride(0)
    if log_norm is not None:
        r.log_norm = log_norm.data_ptr()
    if weight is not None:
        r.weight, r.weight_stride = weight.data_ptr(), weight_stride
    r.logits_type, r.teacher_type = _FLOATS[logits.dtype], _FLOATS[teacher.dtype]
    r.ids_type = _INDEXES[ids.dtype]
    r.temperature = temperature
    r.hip_stream = torch.cuda.current_stream(device).cuda_stream
    return r


def _check_distill(logits, ids, teacher, temperature, log_norm):
    _tensor(logits, "logits", 2, _FLOATS)
    device, n = logits.device, logits.size(0)
    if logits.size(1) < 1:
        raise ValueError("logits: at least one class needed")
    _tensor(ids, "ids", 2, _INDEXES, device)
    _tensor(teacher, "teacher", 2, _FLOATS, device)
    _shape(ids, "ids", (n, ids.size(1)))
    _shape(teacher, "teacher", ids.shape)
    if log_norm is not None:
        _tensor(log_norm, "log_norm", 1, (torch.float32,), device)
        _shape(log_norm, "log_norm", (n,))
    for x, name in ((teacher, "teacher"), (log_norm, "log_norm")):
        if x is not None and x.requires_grad:
            raise ValueError("%s: the teacher is a constant (call .detach())" % name)


def _gradient_like(logits):
    """Rows as far apart as the logits', so that both start alike within 16 bytes; not where that
    would take twice the room."""
    n, v = logits.shape
    stride = logits.stride(0) if n > 1 else v
    if not v < stride <= 2 * v:
        return torch.empty(n, v, dtype=logits.dtype, device=logits.device)
    return torch.empty((n, stride), dtype=logits.dtype, device=logits.device)[:, :v]


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, teacher, log_norm, temperature):
        L = lda.load_library()
        with _On(logits.device):
            r = _distill_rows(logits, ids, teacher, temperature, log_norm)
            loss = torch.empty(r.rows, dtype=torch.float32, device=logits.device)
            stats = torch.empty((r.rows, 8) if ctx.needs_input_grad[0] else 0, dtype=torch.float32,
                                device=logits.device)
            w = _workspace(r, _check(L.lda_distill_workspace(C.byref(r))), logits.device)
            _check(L.lda_distill_loss(C.byref(r), loss.data_ptr(), stats.data_ptr() or None))
            del w
        ctx.save_for_backward(logits, ids, teacher, log_norm, stats)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, upstream):
        logits, ids, teacher, log_norm, stats = ctx.saved_tensors
        L = lda.load_library()
        with _On(logits.device):
            grad = _gradient_like(logits)
            r = _distill_rows(logits, ids, teacher, ctx.temperature, log_norm, upstream,
                              upstream.stride(0))
            _check(L.lda_distill_grad(C.byref(r), stats.data_ptr(), grad.data_ptr(), grad.stride(0)))
        return grad, None, None, None, None


def distill_loss(logits, ids, teacher, *, temperature=1.0, log_norm=None):
    """Loss of every row, float32 [rows], differentiable in logits.

    logits [rows, classes] float32, float16 or bfloat16; ids [rows, slots] int32 or int64, a slot
    whose id is outside [0, classes) is empty; teacher [rows, slots], its logits there.
    Without log_norm the teacher's masses are a softmax over a row's slots; with log_norm, float32
    [rows], they are exp(teacher / temperature - log_norm) and what they leave of 1 is spread evenly over
    the classes without a slot.  The loss is temperature^2 KL(teacher || softmax(logits / temperature)).
    Rows of a tensor may lie any distance apart; within a row elements are adjacent.
    """
    _check_distill(logits, ids, teacher, temperature, log_norm)
    return _Distill.apply(logits, ids, teacher, log_norm, float(temperature))


def distill_loss_and_grad(logits, ids, teacher, *, temperature=1.0, log_norm=None, weight=None):
    """(loss of every row, gradient of sum(weight * loss) in the logits' type), in one call.

    weight: float32 [rows], None: ones.  Rows of weight 0 are left out: loss and gradient 0, whatever
    their logits hold.  Use logits.backward(gradient) to go on from there.
    """
    _check_distill(logits, ids, teacher, temperature, log_norm)
    logits = logits.detach()
    if weight is not None:
        _tensor(weight, "weight", 1, (torch.float32,), logits.device, spread=True)
        _shape(weight, "weight", (logits.size(0),))
    L = lda.load_library()
    with _On(logits.device):
        r = _distill_rows(logits, ids, teacher, float(temperature), log_norm, weight,
                          0 if weight is None else weight.stride(0))
        loss = torch.empty(r.rows, dtype=torch.float32, device=logits.device)
        grad = _gradient_like(logits)
        w = _workspace(r, _check(L.lda_distill_workspace(C.byref(r))), logits.device)
        _check(L.lda_distill_step(C.byref(r), loss.data_ptr(), grad.data_ptr(), grad.stride(0)))
        del w
    return loss, grad


def verify_drafts(target, draft, tokens, accept_u, draw_u, *, lengths=None):
    """(accepted int32 [sequences], tokens [sequences, steps + 1]) of drafted tokens.

    target [sequences, steps + 1, classes] and draft [sequences, steps, classes] hold probabilities,
    float32, float16 or bfloat16; tokens [sequences, steps] int32 or int64 were drawn from draft; accept_u
    [sequences, steps] and draw_u [sequences], float32 in [0, 1), decide.  lengths, int32 [sequences]:
    the drafts each sequence has (None: all).  A row of the result is the accepted drafts, one token drawn
    from what the target has left (or from its next row), then -1.  With steps = 0 the call draws
    one token from every row of target.
    """
    _tensor(target, "target", 3, _FLOATS)
    device = target.device
    B, T, V = target.size(0), _int32(target.size(1) - 1, "steps"), target.size(2)
    if T < 0 or V < 1:
        raise ValueError("target must have steps + 1 rows of at least one class")
    _tensor(draft, "draft", 3, (target.dtype,), device)
    _shape(draft, "draft", (B, T, V))
    _tensor(tokens, "tokens", 2, _INDEXES, device)
    _shape(tokens, "tokens", (B, T))
    _tensor(accept_u, "accept_u", 2, (torch.float32,), device)
    _shape(accept_u, "accept_u", (B, T))
    _tensor(draw_u, "draw_u", 1, (torch.float32,), device)
    _shape(draw_u, "draw_u", (B,))
    if lengths is not None:
        _tensor(lengths, "lengths", 1, (torch.int32,), device)
        _shape(lengths, "lengths", (B,))
    L = lda.load_library()
    with _On(device):
        r = lda.lda_draft_rows()
        r.sequences, r.steps, r.classes = B, T, V
        r.target = target.data_ptr()
        r.target_sequence_stride, r.target_row_stride = target.stride(0), target.stride(1)
        r.draft = draft.data_ptr()
        r.draft_sequence_stride, r.draft_row_stride = draft.stride(0), draft.stride(1)
        r.tokens, r.tokens_stride = tokens.data_ptr(), tokens.stride(0)
        r.lengths = None if lengths is None else lengths.data_ptr()
        r.accept_u, r.accept_u_stride = accept_u.data_ptr(), accept_u.stride(0)
        r.draw_u = draw_u.data_ptr()
        r.probs_type, r.tokens_type = _FLOATS[target.dtype], _INDEXES[tokens.dtype]
        r.hip_stream = torch.cuda.current_stream(device).cuda_stream
        accepted = torch.empty(B, dtype=torch.int32, device=device)
        out = torch.empty(B, T + 1, dtype=tokens.dtype, device=device)
        w = _workspace(r, _check(L.lda_verify_workspace(C.byref(r))), device)
        _check(L.lda_verify_drafts(C.byref(r), accepted.data_ptr(), out.data_ptr(), out.stride(0)))
        del w
    return accepted, out


def _teacher_rows(n, slots, device):
    return (torch.empty(n, slots, dtype=torch.int32, device=device),
            torch.empty(n, slots, dtype=torch.float32, device=device),
            torch.empty(n, dtype=torch.float32, device=device))


def top_topics(z, doc_offsets, K, slots, alpha, *, docs=None):
    """(ids int32 [n, slots], logits float32 [n, slots], log_norm float32 [n]) of documents.

    z int32 [tokens] holds a topic a token, document d those in [doc_offsets[d], doc_offsets[d + 1])
    (int32 or int64).  A row has the document's most frequent topics first, ties to the lower topic,
    with log(count + alpha); empty slots have id -1 and -infinity.  log_norm is log(L + K alpha).  docs,
    int32: the documents wanted, in this order (None: all).
    """
    _tensor(z, "z", 1, (torch.int32,))
    device = z.device
    _tensor(doc_offsets, "doc_offsets", 1, _INDEXES, device)
    if doc_offsets.numel() < 1:
        raise ValueError("doc_offsets must have documents + 1 entries")
    if docs is not None:
        _tensor(docs, "docs", 1, (torch.int32,), device)
    L = lda.load_library()
    with _On(device):
        r = lda.lda_topic_rows()
        r.documents = doc_offsets.numel() - 1
        r.rows = r.documents if docs is None else docs.numel()
        r.docs = None if docs is None else docs.data_ptr()
        r.offsets, r.offsets_type = doc_offsets.data_ptr(), _INDEXES[doc_offsets.dtype]
        r.K, r.z, r.tokens = _int32(K, "K"), z.data_ptr(), z.numel()
        r.slots, r.alpha = _int32(slots, "slots"), float(alpha)
        r.hip_stream = torch.cuda.current_stream(device).cuda_stream
        ids, logits, log_norm = _teacher_rows(r.rows, max(r.slots, 0), device)
        _check(L.lda_top_topics(C.byref(r), ids.data_ptr(), logits.data_ptr(), log_norm.data_ptr()))
    return ids, logits, log_norm


def doc_topics(sampler, slots, docs=None):
    """Lda.doc_topics: top_topics of a sampler's current assignment."""
    device = torch.device("cuda", torch.cuda.current_device())
    slots = _int32(slots, "slots")
    if docs is not None:
        _tensor(docs, "docs", 1, (torch.int32,), device)
    n = sampler.D if docs is None else docs.numel()
    current = torch.cuda.current_stream(device)
    own = torch.cuda.ExternalStream(sampler.stream, device=device) if sampler.stream else \
        torch.cuda.default_stream(device)
    ids, logits, log_norm = _teacher_rows(n, max(slots, 0), device)
    if own != current:  # docs may still be on their way, and the outputs' memory in use
        own.wait_stream(current)
    sampler._ck(lda.load_library().lda_doc_topics(
        sampler._h, n, None if docs is None else docs.data_ptr(), slots, ids.data_ptr(),
        logits.data_ptr(), log_norm.data_ptr()))
    if own != current:
        current.wait_stream(own)
    return ids, logits, log_norm
