"""A classifying head and what is read off it: plain forms, and the work they are timed on.

Three operators that belong together.  `rms_norm` adds the residual and norms hidden rows, in the
inputs' type with its gradient, or to 8 bits with a scale a row; `int8_matmul` multiplies such rows
by the classes' weights, 8-bit integers with a scale a class, to logits; `token_log_probs` gives the
log probabilities of tokens, the entropy of every row, with their gradient, and the top alternatives.

The plain forms are elementary torch operations in 32 bits.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_MOST_NORM = 16_384 * 8_192            # elements of the largest norm
_MOST_PRODUCTS = 4_096 * 4_096 * 141_043
_MOST_LOGITS = 2_048 * 141_043         # of the largest training case


# ---- cases -------------------------------------------------------------------------------------

def _norm(name, rows, width, dtype, form="forward", residual="same", weight="same", pad=0):
    case = {"op": "norm", "form": form, "rows": rows, "width": width, "dtype": dtype,
            "residual": residual, "weight": weight, "pad": pad}
    if name:
        case["name"] = name
    return case


def _product(name, rows, width, classes, dtype, form="product", pad=0):
    case = {"op": "product", "form": form, "rows": rows, "width": width, "classes": classes,
            "dtype": dtype, "pad": pad}
    if name:
        case["name"] = name
    return case


def _log_probs(name, rows, classes, dtype, form="score", top=0, temperature=1.0, masked=0.0,
               padding=0.0, pad=0):
    case = {"op": "log_probs", "form": form, "rows": rows, "classes": classes, "dtype": dtype,
            "top": top, "temperature": temperature, "masked": masked, "padding": padding, "pad": pad}
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one token of one user on its way through a layer: latency alone
        _norm("norm_1x4096_bf16", 1, 4_096, "bf16"),
        # a training step's norm: the sum kept in 32 bits, forward and backward
        _norm("norm_train_8192x4096_bf16", 8_192, 4_096, "bf16", form="train", residual="f32",
              weight="f32"),
        # prompts of a serving batch, to 8 bits for the product behind it
        _norm("norm_8bit_16384x8192_bf16", 16_384, 8_192, "bf16", form="e4m3"),
        # the larger vocabulary of the paper's Table 1 for one user's next token
        _product("product_1x4096x141043_f32", 1, 4_096, 141_043, "f32"),
        # a server's batch over the smaller vocabulary of that table
        _product("product_48x5120x101636_bf16", 48, 5_120, 101_636, "bf16"),
        # hidden rows of a batch of documents to the logits of 10 000 topics: norm, 8 bits, product
        _product("head_2048x4096x10000_bf16", 2_048, 4_096, 10_000, "bf16", form="head"),
        # a teacher's logits for one batch of words, the largest product
        _product("product_4096x4096x141043_bf16", 4_096, 4_096, 141_043, "bf16"),
        # a decision among the topics of a small collection: latency alone
        _log_probs("log_probs_1x1000_f32_top8", 1, 1_000, "f32", top=8),
        # a server's batch reports the alternatives of each drawn token, some classes masked
        _log_probs("log_probs_64x141043_bf16_top20", 64, 141_043, "bf16", top=20, temperature=0.8,
                   masked=0.02),
        # a teacher's rows for distillation: the top 64 of many
        _log_probs("log_probs_2048x101636_f16_top64", 2_048, 101_636, "f16", top=64),
        # a held-out set is scored over a million classes
        _log_probs("log_probs_48x1000000_f32", 48, 1_000_000, "f32"),
        # a training step on log probabilities and entropy, some rows padding
        _log_probs("log_probs_train_2048x141043_bf16", 2_048, 141_043, "bf16", form="train",
                   padding=0.03),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "product", "product", "log_probs", "log_probs", "log_probs"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    pad = rng.choice([0, 0, 0, 24])
    if op == "norm":
        width = _log_int(rng, 64, 16_384)
        if rng.random() < 0.5:
            width = max(64, width // 64 * 64)
        form = rng.choice(["forward", "train", "int8", "e4m3"])
        most = _MOST_NORM // (4 if form == "train" or dtype == "f32" else 1) // width
        rows = _log_int(rng, 1, max(1, min(16_384, most)))
        return _norm(None, rows, width, dtype, form, rng.choice(["none", "same", "f32"]),
                     rng.choice(["none", "same", "f32"]), pad)
    if op == "product":
        rows, width = _log_int(rng, 1, 4_096), _log_int(rng, 64, 16_384)
        if rng.random() < 0.7:
            width = max(64, width // 64 * 64)
        most = min(141_043, _MOST_PRODUCTS // (2 * rows * width), 2_000_000_000 // width)
        classes = _log_int(rng, 64, max(64, most))
        if rng.random() < 0.3:
            return _product(None, rows, width, classes, rng.choice(["f16", "bf16"]), "head", pad)
        return _product(None, rows, width, classes, dtype, "product", pad)
    classes = _log_int(rng, 100, 1_000_000)
    form = rng.choice(["score", "score", "train"])
    most = _MOST_LOGITS // (4 if dtype == "f32" else 2) // classes
    rows = _log_int(rng, 1, max(1, min(2_048, most)))
    top = _log_int(rng, 1, min(256, classes)) if form == "score" and rng.random() < 0.7 else 0
    return _log_probs(None, rows, classes, dtype, form, top, rng.choice([0.7, 1.0, 1.0, 2.0]),
                      rng.choice([0.0, 0.0, 0.3]), rng.choice([0.0, 0.1]), pad)


# ---- inputs ------------------------------------------------------------------------------------

def _random(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(n, width, dtype, pad, g, scale=1.0):
    """Normal numbers, rows of a wider buffer where there is a pad."""
    x = torch.zeros(n, width + pad, dtype=dtype, device="cuda")[:, :width]
    step = max(1, (1 << 27) // width)
    for i in range(0, n, step):
        m = min(step, n - i)
        x[i:i + m] = torch.randn(m, width, generator=g, device="cuda") * scale
    return x


def _hidden(n, width, dtype, pad, g):
    """Hidden rows: each of its own size, a few channels far larger than the others."""
    size = torch.exp(torch.randn(n, 1, generator=g, device="cuda") * 0.5)
    channel = torch.ones(width, device="cuda")
    channel[torch.randint(0, width, (max(1, width // 500),), generator=g, device="cuda")] = 12.0
    return _rows(n, width, dtype, pad, g, size[:min(n, 1)] * channel)


def _prepare_norm(case, g):
    n, width = case["rows"], case["width"]
    dtype = _TYPES[case["dtype"]]
    state = {"x": _hidden(n, width, dtype, case["pad"], g), "residual": None, "weight": None, "eps": 1e-6}
    kind = {"same": dtype, "f32": torch.float32}
    if case["residual"] != "none":
        state["residual"] = _hidden(n, width, kind[case["residual"]], case["pad"], g)
    if case["weight"] != "none":
        state["weight"] = (torch.rand(width, generator=g, device="cuda") + 0.5).to(kind[case["weight"]])
    if case["form"] == "train":
        state["y_grad"] = _rows(n, width, dtype, 0, g, 0.1)
        for name in ("x", "residual", "weight"):
            if state[name] is not None:
                state[name].requires_grad_(True)
        if case["residual"] != "none":
            state["h_grad"] = _rows(n, width, state["residual"].dtype, 0, g, 0.1)
    return state


def _integers(n, width, pad, g):
    x = torch.zeros(n, width + pad, dtype=torch.int8, device="cuda")[:, :width]
    step = max(1, (1 << 27) // width)
    for i in range(0, n, step):
        m = min(step, n - i)
        part = torch.randn(m, width, generator=g, device="cuda") * 32.0
        x[i:i + m] = part.round_().clamp_(-127, 127).to(torch.int8)
    return x


def _prepare_product(case, g):
    n, width, classes = case["rows"], case["width"], case["classes"]
    dtype = _TYPES[case["dtype"]]
    state = {"b": _integers(classes, width, case["pad"], g), "dtype": dtype,
             "b_scale": (torch.rand(classes, generator=g, device="cuda") + 0.5) * 2e-3 / math.sqrt(width)}
    if case["form"] == "head":
        state["x"] = _hidden(n, width, dtype, 0, g)
        state["residual"] = _hidden(n, width, dtype, 0, g)
        state["weight"] = (torch.rand(width, generator=g, device="cuda") + 0.5).to(dtype)
        state["eps"] = 1e-6
    else:
        state["a"] = _integers(n, width, case["pad"], g)
        state["a_scale"] = (torch.rand(n, generator=g, device="cuda") + 0.5) * 0.03
    return state


def _prepare_log_probs(case, g):
    n, classes = case["rows"], case["classes"]
    logits = _rows(n, classes, _TYPES[case["dtype"]], case["pad"], g, 2.5)
    tokens = torch.randint(0, classes, (n,), generator=g, device="cuda")
    if case["masked"]:  # of a grammar: the same classes in every row, in no order
        out = torch.rand(classes, generator=g, device="cuda") < case["masked"]
        out[tokens] = False
        logits.masked_fill_(out, -math.inf)
    # the tokens were drawn from rows like these: most of them are likely ones
    lift = (torch.rand(n, 1, generator=g, device="cuda") * 12.0).to(logits.dtype)
    logits.scatter_(1, tokens[:, None], lift)
    state = {"logits": logits, "tokens": tokens, "temperature": case["temperature"], "top": case["top"]}
    if case["padding"]:
        state["tokens"] = torch.where(torch.rand(n, generator=g, device="cuda") < case["padding"], -1, tokens)
    if case["form"] == "train":
        logits.requires_grad_(True)
        scale = 1024.0 if case["dtype"] == "f16" else 1.0  # half precision with its loss scaled up
        used = (state["tokens"] >= 0).float() * scale
        # advantages of either sign, and a small bonus for entropy; padding has neither
        state["log_prob_grad"] = torch.randn(n, generator=g, device="cuda") * used
        state["entropy_grad"] = torch.full((n,), 0.01, device="cuda") * used
    return state


def prepare(case, seed):
    make = {"norm": _prepare_norm, "product": _prepare_product, "log_probs": _prepare_log_probs}
    state = make[case["op"]](case, _random(seed))
    state["op"], state["form"] = case["op"], case["form"]
    return state


# ---- one pass ----------------------------------------------------------------------------------

def _plain_sum(s):
    """The sum with the residual, as it is handed on."""
    x, r = s["x"].detach(), s["residual"]
    return x if r is None else (x.float() + r.detach().float()).to(r.dtype)


def _plain_norm(s):
    h = _plain_sum(s)
    h32 = h.float()
    inv = torch.rsqrt(h32.square().mean(1, keepdim=True) + s["eps"])
    n = h32 * inv
    return h, n, inv, n if s["weight"] is None else n * s["weight"].detach().float()


def _plain_8bit(y, most):
    scale = y.abs().amax(1, keepdim=True) / most
    return torch.where(scale > 0, y / scale, 0.0), scale


def _plain_norm_pass(s):
    h, n, inv, y = _plain_norm(s)
    with_sum = () if s["residual"] is None else (h,)
    if s["form"] == "e4m3":
        q, scale = _plain_8bit(y, 448.0)
        return (q.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale[:, 0]) + with_sum
    if s["form"] == "int8":  # as the numbers that they stand for
        q, scale = _plain_8bit(y, 127.0)
        return ((q.round() * scale).to(torch.bfloat16), scale[:, 0]) + with_sum
    y = y.to(s["x"].dtype)
    if s["form"] == "forward":
        return (y,) + with_sum
    gy = s["y_grad"].float()
    u = gy if s["weight"] is None else gy * s["weight"].detach().float()
    g = inv * (u - n * (u * n).mean(1, keepdim=True))
    out = (y,) + with_sum
    if s["residual"] is not None:
        g = g + s["h_grad"].float()
    out += (g.to(s["x"].dtype),)
    if s["residual"] is not None:
        out += (g.to(h.dtype),)
    if s["weight"] is not None:
        out += ((gy * n).sum(0).to(s["weight"].dtype),)
    return out


def _plain_product(s):
    if s["form"] == "head":
        h, _, _, y = _plain_norm(s)
        a, scale = _plain_8bit(y, 127.0)
        a = a.round()
    else:
        h, a, scale = None, s["a"].float(), s["a_scale"][:, None]
    y = (torch.matmul(a, s["b"].float().t()) * scale * s["b_scale"]).to(s["dtype"])
    return y if h is None else (y, h)


def _plain_log_probs(s):
    x, t = s["logits"].detach().float(), s["tokens"]
    tau, k = s["temperature"], s["top"]
    n, classes = x.shape
    m = x.amax(1, keepdim=True)
    log_p = (x - m) / tau
    e = torch.exp(log_p)
    total = e.sum(1, keepdim=True)
    log_p -= torch.log(total)
    e /= total
    term = torch.where(e > 0, e * log_p, 0.0)
    entropy = -term.sum(1)
    used = (t >= 0) & (t < classes)
    at = t.clamp(0, classes - 1)[:, None]
    log_prob = torch.where(used, log_p.gather(1, at)[:, 0], 0.0)
    if s["form"] == "train":
        lg, hg = s["log_prob_grad"][:, None], s["entropy_grad"][:, None]
        lg = torch.where(used[:, None], lg, 0.0)
        g = -(lg + hg * entropy[:, None]) * e - hg * term
        g.scatter_add_(1, at, lg)
        return log_prob, entropy, (g / tau).to(s["logits"].dtype)
    if k == 0:
        return log_prob, entropy
    # the largest, equal ones by class: a stable sort
    value, ids = torch.sort(x, dim=1, descending=True, stable=True)
    value, ids = value[:, :k], ids[:, :k]
    none = torch.isinf(value)
    top = torch.where(none, -math.inf, log_p.gather(1, ids))
    return log_prob, entropy, torch.where(none, -1, ids).to(torch.int32), top


def _own(s):
    from paper_1412_1576_amd import operators
    if s["op"] == "norm":
        kw = {"residual": s["residual"], "eps": s["eps"]}
        if s["form"] == "e4m3":
            return operators.rms_norm_8bit(s["x"], s["weight"], dtype=torch.float8_e4m3fn, **kw)
        if s["form"] == "int8":
            q, *rest = operators.rms_norm_8bit(s["x"], s["weight"], dtype=torch.int8, **kw)
            return ((q.float() * rest[0][:, None]).to(torch.bfloat16), *rest)
        y = operators.rms_norm(s["x"], s["weight"], **kw)
        y = y if isinstance(y, tuple) else (y,)
        if s["form"] == "forward":
            return y
        leaves = [s[name] for name in ("x", "residual", "weight") if s[name] is not None]
        grads = [s["y_grad"], s["h_grad"]][:len(y)] if len(y) > 1 else [s["y_grad"]]
        return tuple(v.detach() for v in y) + torch.autograd.grad(y, leaves, grads)
    if s["op"] == "product":
        if s["form"] == "head":
            q, scale, h = operators.rms_norm_8bit(s["x"], s["weight"], residual=s["residual"], eps=s["eps"])
            return operators.int8_matmul(q, scale, s["b"], s["b_scale"], dtype=s["dtype"]), h
        return operators.int8_matmul(s["a"], s["a_scale"], s["b"], s["b_scale"], dtype=s["dtype"])
    if s["form"] == "train":
        log_prob, entropy = operators.token_log_probs(s["logits"], s["tokens"], temperature=s["temperature"])
        grad, = torch.autograd.grad((log_prob, entropy), s["logits"], (s["log_prob_grad"], s["entropy_grad"]))
        return log_prob.detach(), entropy.detach(), grad
    return operators.token_log_probs(s["logits"], s["tokens"], temperature=s["temperature"], top=s["top"])


def run(state):
    if own:
        return _own(state)
    if state["op"] == "norm":
        return _plain_norm_pass(state)
    if state["op"] == "product":
        return _plain_product(state)
    return _plain_log_probs(state)


def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}
    d = size[case["dtype"]]
    if case["op"] == "norm":
        cells = case["rows"] * case["width"]
        r = {"none": 0, "same": d, "f32": 4}[case["residual"]]
        out = 1 if case["form"] in ("int8", "e4m3") else d
        w = {"none": 0, "same": d, "f32": 4}[case["weight"]] * case["width"]
        moved = cells * (d + 2 * r + out) + w
        if case["form"] == "train":  # the gradients come in and go out, the sum is read again
            moved += cells * (d + 2 * r + (r or d) + d) + 2 * w
        if case["form"] in ("int8", "e4m3"):
            moved += 4 * case["rows"]
        return {"bytes": moved, "flops": cells * (14 if case["form"] == "train" else 5)}
    if case["op"] == "product":
        n, k, v = case["rows"], case["width"], case["classes"]
        a = n * k * 3 * d if case["form"] == "head" else n * (k + 4)
        return {"bytes": a + v * (k + 4) + n * v * d, "flops": 2 * n * k * v}
    n, v = case["rows"], case["classes"]
    train = case["form"] == "train"
    kept = n * (1.0 - case["padding"]) if train else n
    return {"bytes": n * v * d + (kept * v * d + n * v * d if train else 0) + n * (16 + 8 * case["top"]),
            "flops": n * v * (12 if train else 6)}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _exact_hidden(s, i, j):
    """Rows i to j: the sum, the root of their mean square, the normed row, and that times the weight."""
    h = s["x"].detach()[i:j].double()
    if s["residual"] is not None:
        h = (h + s["residual"].detach()[i:j].double()).to(s["residual"].dtype).double()
    rms = torch.sqrt((h * h).sum(1) / h.shape[1] + s["eps"])[:, None]
    n = h / rms
    return h, rms, n, n * (1.0 if s["weight"] is None else s["weight"].detach().double())


def _exact_levels(y, form):
    most = 448.0 if form == "e4m3" else 127.0
    scale = y.abs().max(dim=1, keepdim=True)[0] / most
    level = y / scale.masked_fill(scale == 0, 1.0)
    if form == "e4m3":  # three bits behind the leading one, 2^-9 at least
        step = torch.exp2(torch.floor(torch.log2(level.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(level / step) * step, scale
    return torch.round(level), scale


def _exact_norm(s, form):
    rows, width = s["x"].shape
    step = max(1, (1 << 25) // width)
    parts, weight_grad = [], torch.zeros(width, dtype=torch.float64, device="cuda")
    for i in range(0, rows, step):
        j = min(rows, i + step)
        h, rms, n, y = _exact_hidden(s, i, j)
        if form in ("int8", "e4m3"):
            level, scale = _exact_levels(y, form)
            out = [level if form == "e4m3" else level * scale, scale[:, 0]]
        else:
            out = [y]
        if s["residual"] is not None:
            out.append(h)
        if form == "train":
            gy = s["y_grad"][i:j].double()
            u = gy * (1.0 if s["weight"] is None else s["weight"].detach().double())
            along = (u * h).sum(1, keepdim=True) / (width * rms * rms)
            g = (u - along * h) / rms
            if s["residual"] is not None:
                g = g + s["h_grad"][i:j].double()
                out.append(g)
            out.append(g)
            weight_grad += (gy * h / rms).sum(0)
        parts.append(out)
    whole = tuple(torch.cat(c) for c in zip(*parts))
    return whole + ((weight_grad,) if form == "train" and s["weight"] is not None else ())


def _exact_product(s, form):
    b, b_scale = s["b"], s["b_scale"].double()
    if form == "head":
        h, _, _, y = _exact_hidden(s, 0, s["x"].shape[0])
        a, a_scale = _exact_levels(y, "int8")
    else:
        a, a_scale = s["a"].double(), s["a_scale"].double()[:, None]
    out = torch.empty(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
    for i in range(0, b.shape[0], 8192):
        out[:, i:i + 8192] = (a @ b[i:i + 8192].double().T.contiguous()) * a_scale * b_scale[i:i + 8192]
    return (out, h) if form == "head" else out


def _exact_log_probs(s, form):
    tau, k, t = float(s["temperature"]), s["top"], s["tokens"]
    rows, classes = s["logits"].shape
    step = max(1, (1 << 26) // classes)
    parts = []
    for i in range(0, rows, step):
        x = s["logits"].detach()[i:i + step].double()
        token = t[i:i + step]
        z = torch.logsumexp(x / tau, 1)
        p = torch.exp(x / tau - z[:, None])
        mean = (p * x.masked_fill(p == 0, 0.0)).sum(1) / tau
        entropy = z - mean
        held = token >= 0
        place = token.masked_fill(~held, 0)[:, None]
        log_prob = (x.gather(1, place)[:, 0] / tau - z).masked_fill(~held, 0.0)
        out = [log_prob, entropy]
        if form == "train":
            lg, hg = s["log_prob_grad"][i:i + step].double(), s["entropy_grad"][i:i + step].double()
            lg = lg * held
            to_mean = x.masked_fill(p == 0, 0.0) / tau - mean[:, None]
            g = p * (-lg[:, None] - hg[:, None] * to_mean)
            g.scatter_add_(1, place, lg[:, None])
            out.append(g / tau)
        elif k:
            # by value in 32 bits, then by class, as one number: 2^20 classes at most
            bits = s["logits"].detach()[i:i + step].float().add(0.0).view(torch.int32).long()
            order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
            key = order * (1 << 20) + (1 << 20) - 1 - torch.arange(classes, device="cuda")
            best = key.topk(k, dim=1)[0]
            ids = (1 << 20) - 1 - best % (1 << 20)
            top = x.gather(1, ids) / tau - z[:, None]
            out += [ids.masked_fill(top == -math.inf, -1), top]
        parts.append(out)
    return tuple(torch.cat(c) for c in zip(*parts))


def exact(case, seed):
    state = prepare(case, seed)
    find = {"norm": _exact_norm, "product": _exact_product, "log_probs": _exact_log_probs}
    return find[case["op"]](state, case["form"])
