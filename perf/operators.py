"""The row operators beside the sampler: what they compute in plain form, and the work they are timed on.

Three operators that belong together.  `top_topics` reads documents' topic counts out of an
assignment as the top logits of a teacher; the distillation loss trains a student with one logit
a class (a topic, a word) on such rows, with its gradient; `verify_drafts` accepts or redraws the
tokens that a cheap draft proposed, against the target's probabilities, from given random numbers.

The plain forms are elementary torch operations in 32 bits, in 64 where sums stand next to a border.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_MOST_ENTRIES = 4096 * 141_043   # logits of the largest distillation case
_MOST_PROBS = 256 * 9 * 141_043  # probabilities of the largest verification case


# ---- cases -------------------------------------------------------------------------------------

def _distill(name, rows, classes, slots, dtype, form="step", temperature=1.0, rest=False, masked=0,
             ragged=False, left_out=0.0, index="i64", pad=0):
    case = {"op": "distill", "form": form, "rows": rows, "classes": classes, "slots": slots,
            "dtype": dtype, "temperature": temperature, "rest": rest, "masked": masked,
            "ragged": ragged, "left_out": left_out, "index": index, "pad": pad}
    if name:
        case["name"] = name
    return case


def _verify(name, sequences, steps, classes, dtype, ragged=False, sharp=3.0):
    case = {"op": "verify", "sequences": sequences, "steps": steps, "classes": classes,
            "dtype": dtype, "ragged": ragged, "sharp": sharp}
    if name:
        case["name"] = name
    return case


def _topics(name, docs, mean, K, slots, alpha, spread="poisson", picked=False):
    case = {"op": "topics", "docs": docs, "mean": float(mean), "K": K, "slots": slots,
            "alpha": alpha, "spread": spread, "picked": picked}
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # a student of the topics of a small collection, one document at a time: latency alone
        _distill("distill_step_1x1000_f32", 1, 1_000, 16, "f32", rest=True, index="i32"),
        # the same in training: a batch of documents over 10 000 topics, the sampler's rows with
        # their even floor
        _distill("distill_step_2048x10000_f32", 2_048, 10_000, 64, "f32", rest=True, ragged=True,
                 index="i32"),
        # one batch of words of a language model over the larger vocabulary of the paper's Table 1, an
        # odd number; a few rows are padding
        _distill("distill_step_4096x141043_bf16", 4_096, 141_043, 64, "bf16", temperature=2.0,
                 left_out=0.02),
        # through autograd: loss forward, gradient backward, over the smaller vocabulary of that
        # table, classes at its end masked
        _distill("distill_autograd_1024x101636_f16", 1_024, 101_636, 32, "f16", form="autograd",
                 temperature=1.5, masked=36, ragged=True),
        # a held-out set is scored: the loss alone, a few rows of a million classes
        _distill("distill_loss_48x1000000_bf16", 48, 1_000_000, 256, "bf16", form="loss"),
        # one user is answered: four drafts against the target
        _verify("verify_1x4_141043_f32", 1, 4, 141_043, "f32"),
        # plain draws, no drafts, a topic for each document of a batch
        _verify("verify_64x0_1000_f32", 64, 0, 1_000, "f32"),
        # a server's batch, sequences with as many drafts as each had ready
        _verify("verify_32x5_100000_bf16", 32, 5, 100_000, "bf16", ragged=True),
        # a large batch
        _verify("verify_256x4_141043_f32", 256, 4, 141_043, "f32"),
        # teacher rows of one batch of documents out of a collection's assignment
        _topics("topics_2048_of_20000_docs", 20_000, 90, 10_000, 64, 0.01, picked=True),
        # of a whole collection of the NYTimes' shape
        _topics("topics_300000_docs", 300_000, 330, 1_000, 32, 0.05),
        # of books: few documents, long and uneven
        _topics("topics_301_long_docs", 301, 40_000, 100_000, 256, 0.01, spread="wide"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["distill", "distill", "verify", "verify", "topics"])
    if op == "distill":
        classes = _log_int(rng, 100, 1_000_000)
        rows = _log_int(rng, 1, max(1, min(4_096, _MOST_ENTRIES // classes)))
        form = rng.choice(["step", "step", "autograd", "loss"])
        dtype = rng.choice(["f32", "f16", "bf16"])
        if dtype == "f32":
            rows = max(1, rows // 2)
        if form == "autograd":
            rows = max(1, rows // 2)
        rest = rng.random() < 0.4
        return _distill(None, rows, classes, _log_int(rng, 1, 256 if classes >= 512 else 64), dtype,
                        form, rng.choice([0.7, 1.0, 1.0, 2.0, 4.0]), rest,
                        0 if rest else rng.choice([0, 0, classes // 50]), rng.random() < 0.5,
                        rng.choice([0.0, 0.0, 0.1]), rng.choice(["i32", "i64"]), rng.choice([0, 0, 24]))
    if op == "verify":
        classes = _log_int(rng, 100, 1_000_000)
        steps = rng.randint(0, 8)
        most = max(1, _MOST_PROBS // (classes * (2 * steps + 1)))
        return _verify(None, _log_int(rng, 1, min(256, most)), steps, classes,
                       rng.choice(["f32", "f16", "bf16"]), rng.random() < 0.5,
                       rng.choice([1.0, 3.0, 6.0]))
    mean = _log_int(rng, 1, 40_000)
    K = _log_int(rng, 10, 1_000_000)
    return _topics(None, _log_int(rng, 1, max(1, min(200_000, 12_000_000 // mean))), mean, K,
                   _log_int(rng, 1, min(K, 256)), rng.choice([0.01, 0.05, 0.1]),
                   rng.choice(["poisson", "wide"]), rng.random() < 0.3)


# ---- inputs ------------------------------------------------------------------------------------

def _random(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _prepare_distill(case, g):
    N, V, k = case["rows"], case["classes"], case["slots"]
    dtype = _TYPES[case["dtype"]]
    # (rows of a wider buffer where the classes are padded)
    logits = torch.zeros(N, V + case["pad"], dtype=dtype, device="cuda")[:, :V]
    step = max(1, (1 << 27) // V)
    for i in range(0, N, step):
        n = min(step, N - i)
        logits[i:i + n] = torch.randn(n, V, generator=g, device="cuda") * 2.0
    usable = V - case["masked"]
    k_ids = min(k, usable)
    # one id from each of k stretches of the classes: distinct, in any order of size
    width = usable // k_ids
    ids = torch.arange(k_ids, device="cuda") * width + torch.randint(
        0, width, (N, k_ids), generator=g, device="cuda")
    teacher = torch.randn(N, k_ids, generator=g, device="cuda") * 1.5 + 4.0
    teacher = teacher.sort(dim=1, descending=True)[0]
    # the student has learned some of it: its logits there go with the teacher's
    part = (0.8 * teacher + torch.randn(N, k_ids, generator=g, device="cuda")).to(dtype)
    logits.scatter_(1, ids, part)
    if case["masked"]:
        logits[:, usable:] = -math.inf
    if k_ids < k:
        pad = torch.full((N, k - k_ids), -1, dtype=ids.dtype, device="cuda")
        ids = torch.cat([ids, pad], 1)
        teacher = torch.cat([teacher, torch.zeros(N, k - k_ids, device="cuda")], 1)
    if case["ragged"]:
        have = torch.randint(0, k + 1, (N, 1), generator=g, device="cuda")
        empty = torch.arange(k, device="cuda") >= have
        ids = ids.masked_fill(empty, -1)
    state = {"logits": logits, "ids": ids.to(torch.int32 if case["index"] == "i32" else torch.int64),
             "teacher": teacher, "temperature": case["temperature"], "log_norm": None}
    if case["rest"]:
        held = torch.where(ids >= 0, teacher.double() / case["temperature"], -math.inf)
        share = torch.rand(N, generator=g, device="cuda").double() * 0.6 + 0.2  # mass beside the slots
        norm = torch.logsumexp(held, 1) - torch.log1p(-share)
        state["log_norm"] = torch.where(torch.isinf(norm), 0.0, norm).float()
    # the mean over the rows, more or less; half precision with its loss scaled up, as it is trained
    scale = 4096.0 if case["dtype"] == "f16" else 1.0 / N
    weight = (torch.rand(N, generator=g, device="cuda") + 0.5) * scale
    if case["left_out"]:
        weight = weight * (torch.rand(N, generator=g, device="cuda") >= case["left_out"])
    state["weight"] = weight
    return state


def _prepare_verify(case, g):
    B, T, V = case["sequences"], case["steps"], case["classes"]
    dtype = _TYPES[case["dtype"]]
    target = torch.empty(B, T + 1, V, dtype=dtype, device="cuda")
    draft = torch.empty(B, T, V, dtype=dtype, device="cuda")
    tokens = torch.zeros(B, T, dtype=torch.int64, device="cuda")
    for b in range(B):
        x = torch.randn(T + 1, V, generator=g, device="cuda") * case["sharp"]
        target[b] = torch.softmax(x, 1)
        if T:
            x = x[:T] + torch.randn(T, V, generator=g, device="cuda") * 0.7
            draft[b] = torch.softmax(x, 1)
            c = draft[b].double().cumsum(1)
            u = torch.rand(T, 1, generator=g, device="cuda").double() * c[:, -1:]
            tokens[b] = torch.searchsorted(c, u, right=True).clamp_(max=V - 1)[:, 0]
    state = {"target": target, "draft": draft, "tokens": tokens, "lengths": None,
             "accept_u": torch.rand(B, T, generator=g, device="cuda"),
             "draw_u": torch.rand(B, generator=g, device="cuda")}
    if case["ragged"]:
        state["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda",
                                         dtype=torch.int32)
    return state


def _prepare_topics(case, g):
    D, K = case["docs"], case["K"]
    if case["spread"] == "poisson":
        length = torch.poisson(torch.full((D,), case["mean"], device="cuda"), generator=g)
    else:
        length = case["mean"] * torch.exp(torch.randn(D, generator=g, device="cuda") - 0.5)
    length = length.long()
    most = 2 * int(case["mean"] * D) + 64
    offsets = torch.zeros(D + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = length.cumsum(0).clamp_(max=most)
    n = int(offsets[-1])
    doc = torch.repeat_interleave(torch.arange(D, device="cuda"), offsets[1:] - offsets[:-1])
    # a token has one of its document's few topics (the first ones more often), or any
    few = torch.randint(0, K, (D, 12), generator=g, device="cuda", dtype=torch.int32)
    pick = (torch.rand(n, generator=g, device="cuda").square() * 12).long().clamp_(max=11)
    z = few[doc, pick]
    stray = torch.rand(n, generator=g, device="cuda") < 0.2
    z = torch.where(stray, torch.randint(0, K, (n,), generator=g, device="cuda", dtype=torch.int32), z)
    state = {"z": z, "offsets": offsets, "K": K, "slots": case["slots"], "alpha": case["alpha"],
             "docs": None}
    if case["picked"]:
        state["docs"] = torch.randint(0, D, (min(2_048, D),), generator=g, device="cuda",
                                      dtype=torch.int32)
    return state


def prepare(case, seed):
    make = {"distill": _prepare_distill, "verify": _prepare_verify, "topics": _prepare_topics}
    state = make[case["op"]](case, _random(seed))
    state["op"] = case["op"]
    if case["op"] == "distill":
        state["form"] = case["form"]
        if case["form"] == "autograd":
            state["logits"].requires_grad_(True)
    return state


# ---- one pass ----------------------------------------------------------------------------------

def _plain_distill(s):
    x = s["logits"].detach().float()
    N, V = x.shape
    tau = s["temperature"]
    used = s["weight"] != 0
    # the student: q, and log q
    m = x.amax(1, keepdim=True)
    m = torch.where(torch.isinf(m) & (m < 0), 0.0, m)
    log_q = (x - m) / tau
    e = torch.exp(log_q)
    total = e.sum(1, keepdim=True)
    log_q -= torch.log(total)
    # the teacher, as a row of V masses
    ids = s["ids"].long()
    full = (ids >= 0) & (ids < V)
    t = torch.where(full, s["teacher"].float(), -math.inf) / tau
    if s["log_norm"] is None:
        tm = t.amax(1, keepdim=True)
        tm = torch.where(torch.isinf(tm), 0.0, tm)
        p = torch.exp(t - tm)
        sum_p = p.sum(1, keepdim=True)
        p = torch.where(sum_p > 0, p / sum_p, 0.0)
        target = torch.zeros_like(x)
    else:
        p = torch.exp(t - s["log_norm"].float()[:, None])
        others = (V - full.sum(1, keepdim=True)).float()
        rest = torch.where(others > 0, (1.0 - p.sum(1, keepdim=True)).clamp(min=0.0) / others, 0.0)
        target = rest.expand(N, V).contiguous()
        # the classes that have a slot start from nothing
        row = torch.arange(N, device=x.device)[:, None].expand_as(ids)
        target[row[full], ids[full]] = 0.0
    target.scatter_add_(1, ids.clamp(0, V - 1), torch.where(full, p, 0.0))
    mass = target.sum(1, keepdim=True)
    term = target * (torch.log(target) - log_q)
    loss = tau * tau * torch.where(target > 0, term, 0.0).sum(1)
    if s["form"] == "loss":
        return loss
    if s["form"] == "step":  # rows of no weight are left out
        loss = torch.where(used, loss, 0.0)
    used = used & (mass[:, 0] > 0)
    e *= mass / total
    e -= target
    e *= (s["weight"] * tau)[:, None]
    e[~used] = 0.0
    return loss, e.to(s["logits"].dtype)


def _plain_verify(s):
    target, draft, x = s["target"], s["draft"], s["tokens"]
    B, T = x.shape
    rows = torch.arange(B, device=target.device)
    n = torch.full((B,), T, device=x.device) if s["lengths"] is None else s["lengths"].long()
    a = torch.zeros(B, dtype=torch.int64, device=x.device)
    if T:
        p = target[:, :T].gather(2, x[:, :, None])[:, :, 0].double()
        q = draft.gather(2, x[:, :, None])[:, :, 0].double()
        ok = (s["accept_u"].double() * q < p) & (torch.arange(T, device=x.device) < n[:, None])
        a = ok.long().cumprod(1).sum(1)
    p = target[rows, a].double()
    mass = p
    if T:
        q = torch.where((a < n)[:, None], draft[rows, a.clamp(max=T - 1)].double(), 0.0)
        mass = (p - q).clamp_(min=0.0)
        mass = torch.where((mass.sum(1) > 0)[:, None], mass, p)
    c = mass.cumsum(1)
    past = (c > s["draw_u"].double()[:, None] * c[:, -1:]) & (mass > 0)
    index = torch.arange(mass.shape[1], device=x.device)
    token = torch.where(past.any(1), past.long().argmax(1), torch.where(mass > 0, index, -1).amax(1))
    out = torch.full((B, T + 1), -1, dtype=torch.int64, device=x.device)
    step = torch.arange(T, device=x.device)
    out[:, :T] = torch.where(step < a[:, None], x, -1)
    out[rows, a] = token
    return a.to(torch.int32), out


def _plain_topics(s):
    z, offsets, K, k = s["z"], s["offsets"], s["K"], s["slots"]
    docs = s["docs"]
    first, last = offsets[:-1], offsets[1:]
    if docs is not None:
        first, last = first[docs.long()], last[docs.long()]
    length = last - first
    D = length.numel()
    row = torch.repeat_interleave(torch.arange(D, device=z.device), length)
    begin = length.cumsum(0) - length
    at = torch.arange(row.numel(), device=z.device) - begin[row] + first[row]
    key, count = torch.unique(row * K + z[at].long(), return_counts=True)
    row, topic = key // K, key % K
    # by document, then by falling count, then by topic (the order of the keys: a stable sort)
    big = z.numel() + 1
    order = torch.sort(row * big + (big - 1 - count), stable=True)[1]
    row, topic, count = row[order], topic[order], count[order]
    have = torch.bincount(row, minlength=D)
    place = torch.arange(row.numel(), device=z.device) - (have.cumsum(0) - have)[row]
    keep = place < k
    ids = torch.full((D, k), -1, dtype=torch.int32, device=z.device)
    logits = torch.full((D, k), -math.inf, device=z.device)
    ids[row[keep], place[keep]] = topic[keep].to(torch.int32)
    logits[row[keep], place[keep]] = torch.log(count[keep].double() + s["alpha"]).float()
    return ids, logits, torch.log(length.double() + K * s["alpha"]).float()


def run(state):
    s = state
    if own:
        from paper_1412_1576_amd import operators
        if s["op"] == "verify":
            return operators.verify_drafts(s["target"], s["draft"], s["tokens"], s["accept_u"],
                                           s["draw_u"], lengths=s["lengths"])
        if s["op"] == "topics":
            return operators.top_topics(s["z"], s["offsets"], s["K"], s["slots"], s["alpha"],
                                        docs=s["docs"])
        kw = {"temperature": s["temperature"], "log_norm": s["log_norm"]}
        if s["form"] == "step":
            return operators.distill_loss_and_grad(s["logits"], s["ids"], s["teacher"],
                                                   weight=s["weight"], **kw)
        if s["form"] == "loss":
            return operators.distill_loss(s["logits"], s["ids"], s["teacher"], **kw)
        loss = operators.distill_loss(s["logits"], s["ids"], s["teacher"], **kw)
        grad, = torch.autograd.grad(loss, s["logits"], s["weight"])
        return loss.detach(), grad
    if s["op"] == "verify":
        return _plain_verify(s)
    if s["op"] == "topics":
        return _plain_topics(s)
    return _plain_distill(s)


def work(case):
    size = 4 if case.get("dtype") == "f32" else 2
    if case["op"] == "distill":
        N, V, k = case["rows"], case["classes"], case["slots"]
        grad = case["form"] != "loss"
        index = 4 if case["index"] == "i32" else 8
        kept = N * (1.0 - case["left_out"]) if case["form"] == "step" else N
        return {"bytes": kept * V * size + (N * V * size if grad else 0) + N * k * (index + 4) + 12 * N,
                "flops": kept * V * (6 if grad else 3)}
    if case["op"] == "verify":
        B, T, V = case["sequences"], case["steps"], case["classes"]
        # about four drafts in five are accepted; a rejected one needs the draft's row too
        n = 0.5 * T if case["ragged"] else T
        rows = 2.0 - 0.8 ** n
        return {"bytes": B * (rows * V * size + n * (2 * size + 12) + (T + 1) * 8 + 8),
                "flops": B * V * rows * 2}
    docs = min(2_048, case["docs"]) if case["picked"] else case["docs"]
    return {"bytes": docs * (case["mean"] * 4 + 16 + case["slots"] * 8 + 4),
            "flops": docs * case["mean"] * 2}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _exact_distill(s):
    tau = float(s["temperature"])
    N, V = s["logits"].shape
    losses, grads = [], []
    step = max(1, (1 << 26) // V)
    for i in range(0, N, step):
        x = s["logits"].detach()[i:i + step].double()
        ids, t = s["ids"][i:i + step].long(), s["teacher"][i:i + step].double()
        n = x.shape[0]
        log_z = torch.logsumexp(x / tau, 1)
        full = ids >= 0
        at = ids.clamp(min=0)
        lp = t / tau
        rest = torch.zeros(n, dtype=torch.float64, device=x.device)
        others = V - full.sum(1)
        if s["log_norm"] is None:
            held = lp.masked_fill(~full, -math.inf)
            lp = lp - torch.logsumexp(held, 1)[:, None]
            lp = torch.where(full.any(1)[:, None], lp, 0.0)
        else:
            lp = lp - s["log_norm"][i:i + step].double()[:, None]
        p = torch.where(full, lp.exp(), 0.0)
        if s["log_norm"] is not None:
            rest = torch.where(others > 0, (1 - p.sum(1)).clamp(min=0) / others.clamp(min=1), 0.0)
        picked = x.gather(1, at) / tau
        loss = torch.where(full, p * (lp - picked + log_z[:, None]), 0.0).sum(1)
        if s["log_norm"] is not None:
            beside = (x / tau).sum(1) - torch.where(full, picked, 0.0).sum(1)
            even = rest * (others * (torch.log(rest.clamp(min=1e-300)) + log_z) - beside)
            loss = loss + torch.where(rest > 0, even, 0.0)
        mass = p.sum(1) + rest * others
        w = s["weight"][i:i + step].double()
        live = (w != 0) & (mass > 0)
        losses.append(loss * tau * tau)
        if s["form"] == "loss":
            continue
        if s["form"] == "step":
            losses[-1] = torch.where(live, losses[-1], 0.0)
        d = torch.exp(x / tau - log_z[:, None]) * mass[:, None] - rest[:, None]
        d.scatter_add_(1, at, torch.where(full, rest[:, None] - p, 0.0))
        grads.append(torch.where(live[:, None], d * (w * tau)[:, None], 0.0))
    return (torch.cat(losses), torch.cat(grads)) if grads else torch.cat(losses)


def _exact_verify(s):
    p_all, q_all = s["target"], s["draft"]
    B, T = s["tokens"].shape
    x, u, v = s["tokens"].cpu().numpy(), s["accept_u"].cpu().numpy(), s["draw_u"].cpu().numpy()
    n = [T] * B if s["lengths"] is None else s["lengths"].tolist()
    accepted, out = np.zeros(B, np.int64), np.full((B, T + 1), -1, np.int64)
    for b in range(B):
        a = 0
        while a < n[b]:
            if not float(u[b, a]) * float(q_all[b, a, x[b, a]]) < float(p_all[b, a, x[b, a]]):
                break
            out[b, a] = x[b, a]
            a += 1
        mass = p_all[b, a].double().cpu().numpy()
        if a < n[b]:
            left = np.maximum(mass - q_all[b, a].double().cpu().numpy(), 0.0)
            mass = left if left.any() else mass
        held = np.flatnonzero(mass > 0)
        c = np.cumsum(mass[held])
        j = int(np.searchsorted(c, float(v[b]) * c[-1], side="right"))
        out[b, a] = held[min(j, len(held) - 1)]
        accepted[b] = a
    return torch.from_numpy(accepted), torch.from_numpy(out)


def _exact_topics_by_tables(s):
    """Every document's whole table of counts, some documents at a time."""
    offsets, K = s["offsets"], s["K"]
    D, step = len(offsets) - 1, max(1, (1 << 26) // s["K"])
    ids, logits = [], []
    for d in range(0, D, step):
        part = offsets[d:d + step + 1]
        doc = torch.arange(len(part) - 1, device=part.device).repeat_interleave(part.diff())
        cell = doc * K + s["z"][part[0]:part[-1]]
        table = torch.bincount(cell, minlength=(len(part) - 1) * K).view(-1, K)
        key = table * K + (K - 1 - torch.arange(K, device=part.device))
        best = key.topk(s["slots"], dim=1)[0]
        count = best // K
        ids.append(torch.where(count > 0, K - 1 - best % K, -1))
        logits.append(torch.where(count > 0, torch.log(count.double() + s["alpha"]), -math.inf))
    return torch.cat(ids), torch.cat(logits), torch.log(offsets.diff().double() + K * s["alpha"])


def _exact_topics(s):
    if s["docs"] is None and (len(s["offsets"]) - 1) * s["K"] <= 1 << 30:
        return _exact_topics_by_tables(s)
    z, offsets = s["z"].cpu().numpy(), s["offsets"].cpu().numpy()
    docs = range(len(offsets) - 1) if s["docs"] is None else s["docs"].tolist()
    ids = np.full((len(docs), s["slots"]), -1, np.int64)
    logits = np.full((len(docs), s["slots"]), -np.inf)
    norm = np.zeros(len(docs))
    for i, d in enumerate(docs):
        topic, count = np.unique(z[offsets[d]:offsets[d + 1]], return_counts=True)
        order = np.lexsort((topic, -count))[:s["slots"]]
        ids[i, :len(order)] = topic[order]
        logits[i, :len(order)] = np.log(count[order] + s["alpha"])
        norm[i] = math.log(offsets[d + 1] - offsets[d] + s["K"] * s["alpha"])
    return torch.from_numpy(ids), torch.from_numpy(logits), torch.from_numpy(norm)


def exact(case, seed):
    if case["op"] == "topics" and not case["picked"] and case["docs"] > 100_000:
        if case["docs"] * case["K"] > 1 << 30:
            return None
    state = prepare(case, seed)
    if case["op"] == "verify":
        return _exact_verify(state)
    if case["op"] == "topics":
        return _exact_topics(state)
    return _exact_distill(state)
