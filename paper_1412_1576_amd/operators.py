"""The library's operators on rows, on torch tensors of the GPU (lda_mi355x.h has their definitions).

  top_topics, Lda.doc_topics   documents' most frequent topics as the top logits of a teacher
  distill_loss                 distillation from a teacher's top logits, with autograd
  distill_loss_and_grad        the same and its gradient in one call, for weights known beforehand
  verify_drafts                drafted tokens accepted or redrawn from given random numbers
  rms_norm                     root-mean-square norm with the residual's addition, with autograd
  rms_norm_8bit                the same to 8 bits with a scale a row
  int8_matmul                  rows times the classes' weights, 8-bit integers with a scale for each row of both
  token_log_probs              log probabilities of tokens, entropy, top alternatives, with autograd

Work goes to torch's current stream of the tensors' device (inputs made on another stream have to
be ready on it); outputs and workspaces come from torch's allocator; no call waits for the GPU, and
all can be captured into a graph.  Wrong shapes, types or devices raise ValueError,
refusals of the library LdaError.
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad

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


def _wants_gradient(*tensors):
    """Whether a derivative is asked for: of leaves, or along tangents of forward mode, which torch.no_grad() leaves on."""
    for t in tensors:
        if t is not None and getattr(t, "requires_grad", False) and torch.is_grad_enabled():
            return True
    if getattr(forward_ad, "_current_level", 0) < 0:  # no tensor has a tangent
        return False
    return any(isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


def _check_norm(x, weight, residual):
    in_x = _tensor(x, "x", 2, _FLOATS)
    device = x.get_device()
    if x.shape[1] < 1:
        raise ValueError("x: at least one element a row needed")
    same = (x.dtype, torch.float32)
    if weight is not None:
        _tensor(weight, "weight", 1, same, device, x.shape[1:])
    in_residual = None if residual is None else _tensor(residual, "residual", 2, same, device, x.shape)
    return device, in_x, in_residual


def _norm_rows(x, in_x, weight, residual, in_residual, eps, device):
    # in the order of the struct's fields
    rows, width = x.shape
    return lda.lda_norm_rows(
        rows, width, _FLOATS[x.dtype], x.data_ptr(), in_x[0],
        None if residual is None else residual.data_ptr(), 0 if residual is None else in_residual[0],
        None if weight is None else weight.data_ptr(), _FLOATS[x.dtype if weight is None else weight.dtype],
        _FLOATS[x.dtype if residual is None else residual.dtype], eps, 0, _raw_stream(device))


def _same(x):
    """An empty tensor of x's size, rows one behind the other."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)


def _norm(x, weight, residual, eps, with_stats):
    """(y, sum or x itself, stats or None)"""
    device, in_x, in_residual = _check_norm(x, weight, residual)
    L = lda.load_library()
    rows, width = x.shape
    with _On(device):
        r = _norm_rows(x, in_x, weight, residual, in_residual, eps, device)
        y = _same(x)
        h = x if residual is None else _same(residual)
        stats = torch.empty((rows, 2), dtype=torch.float32, device=x.device) if with_stats else None
        _check(L.lda_norm(r, y.data_ptr(), width, h.data_ptr(), width, stats.data_ptr() if with_stats else None))
    return y, h, stats


def _rows_of(g):
    """An upstream gradient with adjacent elements."""
    g = g.resolve_neg()
    return g if g.stride(1) == 1 or g.size(1) <= 1 else g.contiguous()


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        y, h, stats = _norm(x, weight, residual, eps, True)
        ctx.save_for_backward(weight, h, stats)
        ctx.summed = residual is not None
        ctx.eps, ctx.x_type = eps, x.dtype
        ctx.set_materialize_grads(False)
        return (y, h) if ctx.summed else y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, y_grad, h_grad=None):
        weight, h, stats = ctx.saved_tensors
        if y_grad is None:  # the sum alone was used
            to_x = None if h_grad is None or not ctx.needs_input_grad[0] else h_grad.to(ctx.x_type)
            return to_x, None, h_grad, None
        L = lda.load_library()
        device = h.get_device()
        rows, width = h.shape
        to_x, to_weight, to_residual, _ = ctx.needs_input_grad
        with _On(device):
            y_grad = _rows_of(y_grad)
            h_grad = None if h_grad is None else _rows_of(h_grad)
            # x is looked at only where there is no residual, and is the sum there
            r = lda.lda_norm_rows(
                rows, width, _FLOATS[y_grad.dtype], h.data_ptr(), h.stride(0),
                h.data_ptr() if ctx.summed else None, 0, None if weight is None else weight.data_ptr(),
                _FLOATS[y_grad.dtype if weight is None else weight.dtype], _FLOATS[h.dtype], ctx.eps, 0,
                _raw_stream(device))
            one = h.dtype == y_grad.dtype  # gradients of x and of the residual are the same
            x_grad = torch.empty((rows, width), dtype=y_grad.dtype, device=h.device) \
                if to_x or one and to_residual else None
            residual_grad = torch.empty((rows, width), dtype=h.dtype, device=h.device) \
                if to_residual and not one else None
            weight_grad = torch.empty(width, dtype=weight.dtype, device=h.device) if to_weight else None
            g = lda.lda_norm_gradients(
                y_grad.data_ptr(), y_grad.stride(0), None if h_grad is None else h_grad.data_ptr(),
                0 if h_grad is None else h_grad.stride(0), h.data_ptr(), h.stride(0), stats.data_ptr(),
                None if x_grad is None else x_grad.data_ptr(), width,
                None if residual_grad is None else residual_grad.data_ptr(), width,
                None if weight_grad is None else weight_grad.data_ptr())
            w = _workspace(g, _check(L.lda_norm_grad_workspace(r)) if to_weight else 0, h.device)
            _check(L.lda_norm_grad(r, g))
            del w
        return x_grad if to_x else None, weight_grad, (x_grad if one else residual_grad) if to_residual else None, None


def rms_norm(x, weight=None, *, residual=None, eps=1e-6):
    """y, or (y, sum) with a residual: y = weight * sum / sqrt(mean of sum^2 over the row + eps), sum = x + residual.

    x [rows, width] float32, float16 or bfloat16; weight [width] and residual [rows, width] of x's type or
    float32.  The sum has the residual's type and y is the norm of the sum as it is written, in x's type.
    Differentiable in x, weight and residual (backward: tangents of forward mode raise NotImplementedError); sums are
    32-bit at least.  Rows of a tensor may lie any distance apart; within a row elements are adjacent.  A backward pass captured
    into a graph must find no eager graph of the same leaves alive.
    """
    eps = float(eps)
    if _wants_gradient(x, weight, residual):
        return _RmsNorm.apply(x, weight, residual, eps)
    y, h, _ = _norm(x, weight, residual, eps, False)
    return y if residual is None else (y, h)


_LEVELS = {torch.int8: 0, torch.float8_e4m3fn: 1}


def rms_norm_8bit(x, weight=None, *, residual=None, eps=1e-6, dtype=torch.int8):
    """(q, scale), or (q, scale, sum) with a residual: rms_norm's y in 8 bits, q [rows, width] int8 or float8_e4m3fn, times
    scale, float32 [rows].

    The scale brings the largest |y| of a row to 127 or 448; q is y / scale, rounded to nearest, ties to even.  A
    row of zeros has scale 0, a row with a NaN or an infinity scale NaN and q 0.  No gradient: tensors that require one are
    refused outside torch.no_grad(), tensors with a tangent of forward mode everywhere.
    """
    if dtype not in _LEVELS:
        raise ValueError("dtype must be torch.int8 or torch.float8_e4m3fn, not %s" % dtype)
    device, in_x, in_residual = _check_norm(x, weight, residual)
    if _wants_gradient(x, weight, residual):
        raise ValueError("rms_norm_8bit has no gradient (call .detach(), or rms_norm)")
    L = lda.load_library()
    rows, width = x.shape
    with _On(device):
        r = _norm_rows(x, in_x, weight, residual, in_residual, eps, device)
        q = torch.empty((rows, width), dtype=dtype, device=x.device)
        scale = torch.empty(rows, dtype=torch.float32, device=x.device)
        h = None if residual is None else _same(residual)
        _check(L.lda_norm_bytes(r, _LEVELS[dtype], q.data_ptr(), width, scale.data_ptr(),
                                None if h is None else h.data_ptr(), width))
    return (q, scale) if h is None else (q, scale, h)


def int8_matmul(a, a_scale, b, b_scale, *, dtype=torch.bfloat16):
    """[rows, classes] of dtype (float32, float16 or bfloat16): (a @ b.T) * a_scale[:, None] * b_scale.

    a [rows, width] and b [classes, width] int8, as rms_norm_8bit gives a and as weights are kept; a_scale float32
    [rows], b_scale float32 [classes].  The sums are exact (width up to 131071), scaled in 32 bits and rounded once.
    Rows of a and b may lie any distance apart (faster where width and distances are multiples of 16).  No
    gradient: scales that require one are refused outside torch.no_grad(), scales with a tangent of forward mode everywhere.
    """
    if dtype not in _FLOATS:
        raise ValueError("dtype must be one of %s, not %s" % (", ".join(map(str, _FLOATS)), dtype))
    in_a = _tensor(a, "a", 2, (torch.int8,))
    device = a.get_device()
    in_b = _tensor(b, "b", 2, (torch.int8,), device)
    rows, width = a.shape
    classes = b.shape[0]
    if b.shape[1] != width:
        raise ValueError("b has %d numbers a row, a %d" % (b.shape[1], width))
    if classes < 1:
        raise ValueError("b: at least one class needed")
    classes = _int32(classes, "classes")
    _tensor(a_scale, "a_scale", 1, (torch.float32,), device, (rows,))
    _tensor(b_scale, "b_scale", 1, (torch.float32,), device, (classes,))
    if _wants_gradient(a_scale, b_scale):
        raise ValueError("int8_matmul has no gradient (call .detach() on the scales)")
    L = lda.load_library()
    with _On(device):
        # in the order of the struct's fields
        r = lda.lda_product_rows(
            rows, classes, width, a.data_ptr(), in_a[0], a_scale.data_ptr(), b.data_ptr(), in_b[0],
            b_scale.data_ptr(), _FLOATS[dtype], 0, None, 0, _raw_stream(device))
        need = _check(L.lda_product_workspace(r))
        out = torch.empty((rows, classes), dtype=dtype, device=a.device)
        w = _workspace(r, need, a.device)
        _check(L.lda_product(r, out.data_ptr(), classes))
        del w
    return out


def _log_prob_rows(logits, tokens, temperature, top):
    # in the order of the struct's fields
    rows, classes = logits.shape
    return lda.lda_log_prob_rows(
        rows, classes, top, logits.data_ptr(), logits.stride(0), tokens.data_ptr(), tokens.stride(0),
        _FLOATS[logits.dtype], _INDEXES[tokens.dtype], temperature, 0, None, 0, _raw_stream(logits.get_device()))


def _log_probs(logits, tokens, temperature, top, with_stats):
    """(log_prob, entropy, ids, log probabilities, stats), the last three None where not wanted"""
    L = lda.load_library()
    device = logits.device
    with _On(logits.get_device()):
        r = _log_prob_rows(logits, tokens, temperature, top)
        need = _check(L.lda_log_probs_workspace(r))
        n = r.rows
        log_prob = torch.empty(n, dtype=torch.float32, device=device)
        entropy = torch.empty_like(log_prob)
        ids = values = stats = None
        if top > 0:
            values = torch.empty((n, top), dtype=torch.float32, device=device)
            ids = torch.empty_like(values, dtype=torch.int32)
        if with_stats:
            stats = torch.empty((n, 4), dtype=torch.float32, device=device)
        w = _workspace(r, need, device)
        _check(L.lda_log_probs(r, log_prob.data_ptr(), entropy.data_ptr(), ids.data_ptr() if top > 0 else None,
                               values.data_ptr() if top > 0 else None, stats.data_ptr() if with_stats else None))
        del w
    return log_prob, entropy, ids, values, stats


class _LogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, temperature, top):
        log_prob, entropy, ids, values, stats = _log_probs(logits, tokens, temperature, top, True)
        ctx.save_for_backward(logits, tokens, stats)
        ctx.temperature = temperature
        ctx.set_materialize_grads(False)
        if top <= 0:
            return log_prob, entropy
        ctx.mark_non_differentiable(ids, values)
        return log_prob, entropy, ids, values

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, log_prob_grad, entropy_grad, *none):
        if log_prob_grad is None and entropy_grad is None:
            return None, None, None, None
        logits, tokens, stats = ctx.saved_tensors
        L = lda.load_library()
        with _On(logits.get_device()):
            grad = _gradient_like(logits)
            r = _log_prob_rows(logits, tokens, ctx.temperature, 0)
            a, b = (None if g is None else g.resolve_neg() for g in (log_prob_grad, entropy_grad))
            _check(L.lda_log_probs_grad(
                r, stats.data_ptr(), None if a is None else a.data_ptr(), 0 if a is None else a.stride(0),
                None if b is None else b.data_ptr(), 0 if b is None else b.stride(0), grad.data_ptr(), grad.stride(0)))
        return grad, None, None, None


def token_log_probs(logits, tokens, *, temperature=1.0, top=0):
    """(log_prob, entropy), float32 [rows]; with top also (ids int32, log probabilities float32), [rows, top].

    logits [rows, classes] float32, float16 or bfloat16; tokens [rows] int32 or int64: log_prob is that of the row's token
    under softmax(logits / temperature), 0 where the token is outside [0, classes) (padding).  top: so many of the
    likeliest classes and their log probabilities, the likeliest first, equal ones by class; slots without a class of
    probability have id -1 and -infinity.  At temperature 1 they are a teacher for distill_loss, with log_norm zeros.
    Differentiable in logits through log_prob and entropy (not through the alternatives; backward: a tangent of forward
    mode raises NotImplementedError); rows whose gradients of both
    are 0 are left out, whatever their logits hold.  A row without any logit above -infinity has log_prob -infinity, entropy 0 and
    gradient 0.  Rows of a tensor may lie any distance apart; within a row elements are adjacent.  A
    backward pass captured into a graph must find no eager graph of the same leaves alive.
    """
    _tensor(logits, "logits", 2, _FLOATS)
    if logits.shape[1] < 1:
        raise ValueError("logits: at least one class needed")
    _tensor(tokens, "tokens", 1, _INDEXES, logits.get_device(), logits.shape[:1], spread=True)
    temperature, top = float(temperature), _int32(top, "top")
    if _wants_gradient(logits):
        return _LogProbs.apply(logits, tokens, temperature, top)
    out = _log_probs(logits, tokens, temperature, top, False)
    return out[:4] if top > 0 else out[:2]
