"""The library's operators on rows, on torch tensors of the GPU (lda_mi355x.h has their definitions).

  top_topics, Lda.doc_topics   documents' most frequent topics as the top logits of a teacher
  distill_loss                 distillation from a teacher's top logits, with autograd
  distill_loss_and_grad        the same and its gradient in one call, for weights known beforehand
  verify_drafts                drafted tokens accepted or redrawn from given random numbers

Work goes to torch's current stream of the tensors' device (inputs made on another stream have to
be ready on it); outputs and workspaces come from torch's allocator; no call waits for the GPU, and
all can be captured into a graph.  Wrong shapes, types or devices raise ValueError,
refusals of the library LdaError.
"""
from __future__ import annotations

import torch

from . import lda
from .lda import LDA_OK, LdaError

_FLOATS = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_INDEXES = {torch.int32: 0, torch.int64: 1}
_INT32 = 2 ** 31 - 1


def _stream_of(device):
    return torch.cuda.current_stream(device).cuda_stream


# What current_stream() wraps, where torch has it: some 1 us less of a call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream_of)


def _tensor(x, name, dims, types, device=None, shape=None, spread=False):
    """The checks of one argument; returns its strides.  A few tests on the way that a right
    call takes: small calls are bound by the host."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError("%s must be a tensor on the GPU" % name)
    if x.dtype not in types:
        raise ValueError("%s must be one of %s, not %s" % (name, ", ".join(map(str, types)), x.dtype))
    size, stride = x.shape, x.stride()
    if len(size) != dims:
        raise ValueError("%s must have %d dimensions, not %d" % (name, dims, len(size)))
    if device is not None and x.get_device() != device:
        raise ValueError("%s is on %s, not on cuda:%d" % (name, x.device, device))
    if shape is not None and size != shape:
        raise ValueError("%s has shape %s, not %s" % (name, tuple(size), tuple(shape)))
    last = size[-1]
    if not spread and stride[-1] != 1 and last > 1:
        raise ValueError("%s: elements of a row must be adjacent (call .contiguous())" % name)
    if last > _INT32 and dims > 1:
        raise ValueError("%s: a row has at most 2^31 - 1 elements" % name)
    if x.is_neg():
        raise ValueError("%s: a view that negates its memory (call .resolve_neg())" % name)
    return stride


def _int32(x, name):
    x = int(x)
    if not -_INT32 <= x <= _INT32:
        raise ValueError("%s does not fit 32 bits" % name)
    return x


def _check(rc):
    if rc < LDA_OK:
        raise LdaError(rc, (lda.load_library().lda_last_error(None) or b"").decode())
    return rc


class _On:
    """A device as the current one, for the length of a call."""

    def __init__(self, device):
        self.device = device

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.device:
            torch.cuda.set_device(self.device)

    def __exit__(self, *exc):
        if self.before != self.device:
            torch.cuda.set_device(self.before)


def _workspace(r, nbytes, device):
    """Room for the call; the caching allocator keeps it from work of other streams."""
    if nbytes == 0:
        return None
    w = torch.empty(nbytes, dtype=torch.uint8, device=device)
    r.workspace, r.workspace_bytes = w.data_ptr(), nbytes
    return w


def _distill_rows(logits, ids, teacher, temperature, log_norm, weight=None, weight_stride=0):
    # in the order of the struct's fields
    rows, classes = logits.shape
    return lda.lda_distill_rows(
        rows, classes, ids.shape[1], logits.data_ptr(), logits.stride(0), ids.data_ptr(), ids.stride(0),
        teacher.data_ptr(), teacher.stride(0), None if log_norm is None else log_norm.data_ptr(),
        None if weight is None else weight.data_ptr(), weight_stride, _FLOATS[logits.dtype],
        _INDEXES[ids.dtype], _FLOATS[teacher.dtype], temperature, None, 0,
        _raw_stream(logits.get_device()))


def _check_distill(logits, ids, teacher, log_norm):
    _tensor(logits, "logits", 2, _FLOATS)
    device = logits.get_device()
    n, classes = logits.shape
    if classes < 1:
        raise ValueError("logits: at least one class needed")
    _tensor(ids, "ids", 2, _INDEXES, device)
    if ids.size(0) != n:
        raise ValueError("ids has %d rows, logits %d" % (ids.size(0), n))
    _tensor(teacher, "teacher", 2, _FLOATS, device, ids.shape)
    if log_norm is not None:
        _tensor(log_norm, "log_norm", 1, (torch.float32,), device, (n,))
    if teacher.requires_grad or log_norm is not None and log_norm.requires_grad:
        raise ValueError("teacher: a constant (call .detach() on it and on log_norm)")
    return device


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
        with _On(logits.get_device()):
            r = _distill_rows(logits, ids, teacher, temperature, log_norm)
            loss = torch.empty(r.rows, dtype=torch.float32, device=logits.device)
            stats = torch.empty((r.rows, 8) if ctx.needs_input_grad[0] else 0, dtype=torch.float32,
                                device=logits.device)
            w = _workspace(r, _check(L.lda_distill_workspace(r)), logits.device)
            _check(L.lda_distill_loss(r, loss.data_ptr(), stats.data_ptr() or None))
            del w
        ctx.save_for_backward(logits, ids, teacher, log_norm, stats)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, upstream):
        logits, ids, teacher, log_norm, stats = ctx.saved_tensors
        L = lda.load_library()
        with _On(logits.get_device()):
            grad = _gradient_like(logits)
            r = _distill_rows(logits, ids, teacher, ctx.temperature, log_norm, upstream,
                              upstream.stride(0))
            _check(L.lda_distill_grad(r, stats.data_ptr(), grad.data_ptr(), grad.stride(0)))
        return grad, None, None, None, None


def distill_loss(logits, ids, teacher, *, temperature=1.0, log_norm=None):
    """Loss of every row, float32 [rows], differentiable in logits.

    logits [rows, classes] float32, float16 or bfloat16; ids [rows, slots] int32 or int64, a slot
    whose id is outside [0, classes) is empty; teacher [rows, slots], its logits there.
    Without log_norm the teacher's masses are a softmax over a row's slots; with log_norm, float32
    [rows], they are exp(teacher / temperature - log_norm) and what they leave of 1 is spread evenly over
    the classes without a slot.  The loss is temperature^2 KL(teacher || softmax(logits / temperature)) where the
    ids of a row differ; a class with several slots has their masses' sum, and the gradient of that, but each slot's
    own p log p in the loss (the term that the student does not change).
    Rows of a tensor may lie any distance apart; within a row elements are adjacent.
    A backward pass captured into a graph must find no eager graph of the same leaves alive (delete losses
    that were computed from them before).
    """
    _check_distill(logits, ids, teacher, log_norm)
    return _Distill.apply(logits, ids, teacher, log_norm, float(temperature))


def distill_loss_and_grad(logits, ids, teacher, *, temperature=1.0, log_norm=None, weight=None):
    """(loss of every row, gradient of sum(weight * loss) in the logits' type), in one call.

    weight: float32 [rows], None: ones.  Rows of weight 0 are left out: loss and gradient 0, whatever
    their logits hold.  Use logits.backward(gradient) to go on from there.
    """
    device = _check_distill(logits, ids, teacher, log_norm)
    spread = 0
    if weight is not None:
        spread, = _tensor(weight, "weight", 1, (torch.float32,), device, logits.shape[:1], spread=True)
    L = lda.load_library()
    with _On(device):
        r = _distill_rows(logits, ids, teacher, temperature, log_norm, weight, spread)
        loss = torch.empty(r.rows, dtype=torch.float32, device=device)
        grad = _gradient_like(logits)
        w = _workspace(r, _check(L.lda_distill_workspace(r)), device)
        _check(L.lda_distill_step(r, loss.data_ptr(), grad.data_ptr(), grad.stride(0)))
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
    in_target = _tensor(target, "target", 3, _FLOATS)
    device = target.get_device()
    B, T, V = target.shape
    T = _int32(T - 1, "steps")
    if T < 0 or V < 1:
        raise ValueError("target must have steps + 1 rows of at least one class")
    in_draft = _tensor(draft, "draft", 3, (target.dtype,), device, (B, T, V))
    in_tokens = _tensor(tokens, "tokens", 2, _INDEXES, device, (B, T))
    in_accept = _tensor(accept_u, "accept_u", 2, (torch.float32,), device, (B, T))
    _tensor(draw_u, "draw_u", 1, (torch.float32,), device, (B,))
    if lengths is not None:
        _tensor(lengths, "lengths", 1, (torch.int32,), device, (B,))
    L = lda.load_library()
    with _On(device):
        # in the order of the struct's fields
        r = lda.lda_draft_rows(
            B, T, V, target.data_ptr(), in_target[0], in_target[1], draft.data_ptr(), in_draft[0], in_draft[1],
            tokens.data_ptr(), in_tokens[0], None if lengths is None else lengths.data_ptr(),
            accept_u.data_ptr(), in_accept[0], draw_u.data_ptr(), _FLOATS[target.dtype],
            _INDEXES[tokens.dtype], None, 0, _raw_stream(device))
        accepted = torch.empty(B, dtype=torch.int32, device=device)
        out = torch.empty(B, T + 1, dtype=tokens.dtype, device=device)
        w = _workspace(r, _check(L.lda_verify_workspace(r)), device)
        _check(L.lda_verify_drafts(r, accepted.data_ptr(), out.data_ptr(), T + 1))
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
    device = z.get_device()
    _tensor(doc_offsets, "doc_offsets", 1, _INDEXES, device)
    documents = doc_offsets.numel() - 1
    if documents < 0:
        raise ValueError("doc_offsets must have documents + 1 entries")
    if docs is not None:
        _tensor(docs, "docs", 1, (torch.int32,), device)
    n = documents if docs is None else docs.numel()
    slots = _int32(slots, "slots")
    L = lda.load_library()
    with _On(device):
        # in the order of the struct's fields
        r = lda.lda_topic_rows(n, None if docs is None else docs.data_ptr(), documents, doc_offsets.data_ptr(),
                               _INDEXES[doc_offsets.dtype], _int32(K, "K"), z.data_ptr(), z.numel(), slots, 0,
                               alpha, None, 0, _raw_stream(device))
        w = _workspace(r, _check(L.lda_topics_workspace(r)), device)
        ids, logits, log_norm = _teacher_rows(n, max(slots, 0), device)
        _check(L.lda_top_topics(r, ids.data_ptr(), logits.data_ptr(), log_norm.data_ptr()))
        del w
    return ids, logits, log_norm


def doc_topics(sampler, slots, docs=None):
    """Lda.doc_topics: top_topics of a sampler's current assignment; captured on the sampler's own stream, of the
    assignment that there is when the graph is replayed."""
    device = sampler.device
    slots = _int32(slots, "slots")
    if docs is not None:
        _tensor(docs, "docs", 1, (torch.int32,), device)
    n = sampler.D if docs is None else docs.numel()
    with _On(device):
        apart = _raw_stream(device) != sampler.stream
        if apart and torch.cuda.is_current_stream_capturing():
            raise ValueError("doc_topics in a captured stream: only where it is the sampler's own stream")
        if apart:
            current = torch.cuda.current_stream(device)
            own = torch.cuda.ExternalStream(sampler.stream, device=device) if sampler.stream else \
                torch.cuda.default_stream(device)
        ids, logits, log_norm = _teacher_rows(n, max(slots, 0), device)
        if apart:  # docs may still be on their way, and the outputs' memory in use
            own.wait_stream(current)
        sampler._ck(lda.load_library().lda_doc_topics(
            sampler._h, n, None if docs is None else docs.data_ptr(), slots, ids.data_ptr(),
            logits.data_ptr(), log_norm.data_ptr()))
        if apart:
            current.wait_stream(own)
    return ids, logits, log_norm
