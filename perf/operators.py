"""Cases and plain forms of the vocabulary-row operators around speculative decoding: the record of a row's top logits, the
distillation of a draft model from that record, beam selection over a draft's vocabulary rows and the reordering of its states.

`run` computes each operator in elementary torch operations while `own` is false, and calls the framework's entry points
(`paper_2405_19715_b200.specdec`) when it is true.  Both take the same inputs and give the same outputs.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}
_handle = None


def listed():
    return [
        # one sequence's verification round: the K + 1 = 5 target rows whose top logits go into the draft's training record
        dict(name="record_round", op="record", rows=5, V=32000, dtype="bf16", k=50, T=1.0, pad=0),
        # a whole batch's round (256 sequences, 17 rows each) at the largest vocabulary of the benchmark
        dict(name="record_batch", op="record", rows=4352, V=128256, dtype="bf16", k=50, T=1.0, pad=0),
        # an odd vocabulary in rows padded to another stride, kept in 32 bits, long lists
        dict(name="record_odd_f32", op="record", rows=300, V=50021, dtype="f32", k=200, T=0.75, pad=3),
        # a few tokens of online distillation between two rounds
        dict(name="step_few", op="step", rows=16, V=32000, dtype="bf16", k=16, T=1.0, pad=0, rest=False, padded=False),
        # a training batch of 4096 tokens at the largest vocabulary: loss and gradient in one call
        dict(name="step_batch", op="step", rows=4096, V=128256, dtype="bf16", k=64, T=1.0, pad=0, rest=True, padded=False),
        # an odd vocabulary, padded stride, half precision, a batch with padding rows, softened by T = 2
        dict(name="step_odd_f16", op="step", rows=511, V=32003, dtype="f16", k=100, T=2.0, pad=5, rest=True, padded=True),
        # loss first, gradient later with the upstream's row gradients, as under a framework's backward pass
        dict(name="loss_then_gradient", op="pair", rows=2048, V=32000, dtype="bf16", k=50, T=1.0, pad=0, rest=True, padded=False),
        # beam search of one sequence: twice as many candidates as beams
        dict(name="beam_one", op="beam", B=1, W=4, V=32000, dtype="bf16", M=8, T=1.0, ends=False),
        # beam search of a serving batch
        dict(name="beam_batch", op="beam", B=128, W=8, V=128256, dtype="bf16", M=16, T=1.0, ends=False),
        # odd sizes, 32 bits, with finished beams and beams that hold nothing yet
        dict(name="beam_odd_f32", op="beam", B=9, W=5, V=50021, dtype="f32", M=10, T=0.75, ends=True),
        # a small draft model's cache of one sequence after a selection
        dict(name="reorder_one", op="reorder", L=8, B=1, W=4, H=4, S=256, D=64, dtype="bf16", longest=131),
        # the caches of a batch (16 layers of keys and values, sequences of different lengths)
        dict(name="reorder_batch", op="reorder", L=32, B=16, W=4, H=8, S=512, D=128, dtype="bf16", longest=500),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["record", "step", "pair", "beam", "reorder"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    T = rng.choice([0.5, 0.75, 1.0, 1.25, 2.0])
    if op == "reorder":
        c = dict(op=op, L=_log_int(rng, 1, 32), B=_log_int(rng, 1, 32), W=rng.randint(2, 16), H=rng.randint(1, 8), S=_log_int(rng, 16, 1024),
                 D=rng.choice([24, 33, 64, 80, 128]), dtype=dtype)
        while c["L"] * c["B"] * c["W"] * c["H"] * c["S"] * c["D"] * _SIZE[dtype] > 1 << 30:
            c["L"] = max(1, c["L"] // 2)
            c["B"] = max(1, c["B"] // 2)
        c["longest"] = rng.randint(1, c["S"])
        return c
    V = _log_int(rng, 1000, 131072)
    if rng.random() < 0.5:
        V = V // 8 * 8
    room = (1 << 30) // (V * _SIZE[dtype])
    if op == "beam":
        W = rng.randint(1, 16)
        return dict(op=op, B=_log_int(rng, 1, max(1, min(64, room // (2 * W)))), W=W, V=V, dtype=dtype, M=rng.randint(1, 2 * W), T=T, ends=rng.random() < 0.5)
    c = dict(op=op, rows=_log_int(rng, 1, min(4096, room // (1 if op == "record" else 2))), V=V, dtype=dtype, k=_log_int(rng, 1, 256), T=T,
             pad=rng.choice([0, 0, 1, 8, 13]))
    if op != "record":
        c |= dict(rest=rng.random() < 0.6, padded=rng.random() < 0.3)
    return c


# ------------------------------------------------------------------------------------------------ inputs


def _rows(g, n, V, pad, dtype):
    """[n, V] logits N(0, 2.5^2); with pad > 0 rows of a wider buffer whose other columns hold NaN."""
    x = torch.empty(n, V + pad, dtype=_TYPES[dtype], device="cuda")
    x[:, V:] = float("nan")
    step = max(1, (1 << 27) // V)
    for at in range(0, n, step):
        part = x[at:at + step, :V]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * 2.5)
    return x[:, :V]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 13)
    c = dict(case)
    op = c["op"]
    if op == "reorder":
        L, B, W, H, S, D = (c[n] for n in "LBWHSD")
        c["cache"] = torch.randn(L, B, W, H, S, D, generator=g, device="cuda", dtype=_TYPES[c["dtype"]])
        c["parents"] = torch.randint(0, W, (B, W), generator=g, device="cuda", dtype=torch.int32)
        c["lens"] = torch.randint(max(1, c["longest"] // 2), c["longest"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        return c
    if op == "beam":
        B, W, V = c["B"], c["W"], c["V"]
        c["logits"] = _rows(g, B * W, V, 0, c["dtype"]).view(B, W, V)
        c["scores"] = torch.randn(B, W, generator=g, device="cuda") * 2 - 12
        c["finished"] = None
        if c["ends"]:
            c["finished"] = (torch.rand(B, W, generator=g, device="cuda") < 0.2).to(torch.int32)
            dead = torch.rand(B, W, generator=g, device="cuda") < 0.2
            dead[:, 0] = False
            c["scores"] = torch.where(dead, float("-inf"), c["scores"])
        return c
    n, V, k = c["rows"], c["V"], c["k"]
    teacher = _rows(g, n, V, c["pad"] if op == "record" else 0, c["dtype"])
    if op == "record":
        c["logits"] = teacher
        return c
    # the record of the teacher's rows, and a student that is near it but not the same
    c["values"] = torch.empty(n, k, device="cuda")
    c["tokens"] = torch.empty(n, k, dtype=torch.int32, device="cuda")
    c["lse"] = torch.empty(n, device="cuda") if c["rest"] else None
    student = torch.full((n, V + c["pad"]), float("nan"), dtype=_TYPES[c["dtype"]], device="cuda")[:, :V]
    step = max(1, (1 << 27) // V)
    for at in range(0, n, step):
        t = teacher[at:at + step].float()
        top = torch.topk(t, k, dim=1)
        c["values"][at:at + step] = top.values
        c["tokens"][at:at + step] = top.indices.to(torch.int32)
        if c["rest"]:
            c["lse"][at:at + step] = torch.logsumexp(t.double() / c["T"], 1).float()
        student[at:at + step].copy_(t + torch.randn(t.shape, generator=g, device="cuda"))
    if c["padded"]:  # every fifth row is padding: an empty list
        c["tokens"][4::5] = -1
    c["logits"] = student
    # 1 / (number of tokens), as a mean over the batch gives, a little different for each row; half precision trains with a loss scale
    c["weight"] = (0.5 + torch.rand(n, generator=g, device="cuda")) / n * (2.0 ** 14 if c["dtype"] == "f16" else 1.0)
    return c


# ------------------------------------------------------------------------------------------------ plain forms


def _record(s):
    x = s["logits"].float()
    bits = x.view(torch.int32) if x.is_contiguous() else x.contiguous().view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64)  # the order of the floats, as whole numbers
    key = (key << 22) - torch.arange(x.shape[1], device=x.device)  # a tie goes to the lower index
    at = torch.topk(key, s["k"], dim=1).indices
    z = x.double() / s["T"] if x.numel() < 1 << 27 else x / s["T"]
    m = z.amax(1, keepdim=True)
    lse = m.double()[:, 0] + (z - m).exp().sum(1).double().log()
    return {"values": x.gather(1, at), "tokens": at.to(torch.int32), "lse": lse.float()}


def _teacher(s):
    """p of the listed tokens, the rest's share and which entries count, in 64 bits (the lists are short)."""
    used = s["tokens"] >= 0
    v = s["values"].double() / s["T"]
    if s["rest"]:
        p = torch.where(used, (v - s["lse"].double()[:, None]).exp(), 0.0)
        rest = (1 - p.sum(1)).clamp(min=0)
    else:
        v = torch.where(used, v, float("-inf"))
        e = torch.where(used, (v - v.amax(1, keepdim=True)).exp(), 0.0)
        total = e.sum(1, keepdim=True)
        p = torch.where(total > 0, e / total, 0.0)
        rest = torch.zeros_like(total[:, 0])
    return p, torch.where(used.any(1), rest, 0.0), used


def _student(s):
    z = s["logits"].float() / s["T"]
    m = z.amax(1, keepdim=True)
    return z, m, (z - m).exp()


def _distill(s):
    """loss [n] and what the gradient needs."""
    z, m, e = _student(s)
    n, V = z.shape
    p, rest, used = _teacher(s)
    at = s["tokens"].clamp(min=0).long()
    total = e.sum(1).double()
    outside = torch.cat([e, e.new_zeros(n, 1)], 1)
    outside.scatter_(1, torch.where(used, at, V), 0.0)
    rest_q = outside.sum(1).double() / total
    del outside
    rest = torch.where(rest_q > 0, rest, 0.0)
    log_q = (z.gather(1, at) - m).double() - total.log()[:, None]
    loss = torch.where(p > 0, p * (p.log() - log_q), 0.0).sum(1) + torch.where(rest > 0, rest * (rest.log() - rest_q.log()), 0.0)
    live = used.any(1)
    return torch.where(live, loss, 0.0).float(), (e, total, p, rest, rest_q, used, at, live)


def _gradient(s, kept, weight):
    e, total, p, rest, rest_q, used, at, live = kept
    n, V = e.shape
    q = e / total.float()[:, None]
    mass = p.sum(1) + rest
    w = torch.where(live, weight.double() / s["T"], 0.0)
    share = torch.where(rest > 0, rest / rest_q, 0.0)
    out = q * (w * (mass - share)).float()[:, None]
    listed_ = (w[:, None] * (mass[:, None] * q.gather(1, at).double() - p)).float()
    out = torch.cat([out, out.new_zeros(n, 1)], 1)
    out.scatter_(1, torch.where(used, at, V), listed_)
    return out[:, :V].to(s["logits"].dtype)


def _beam(s):
    B, W, V = s["logits"].shape
    x = s["logits"].double() / s["T"]
    m = x.amax(2, keepdim=True)
    score = s["scores"].double()[:, :, None] + (x - (m + (x - m).exp().sum(2, keepdim=True).log()))
    if s["finished"] is not None:  # a finished beam offers itself once, through token 0, with the score that it has
        ended = s["finished"].bool()[:, :, None]
        first = torch.arange(V, device=x.device) == 0
        score = torch.where(ended, float("-inf"), score)
        score = torch.where(ended & first, s["scores"].double()[:, :, None], score)
    order = torch.sort(score.view(B, W * V), dim=1, descending=True, stable=True)
    flat = order.indices[:, :s["M"]]
    return {"scores": order.values[:, :s["M"]].float(), "parents": (flat // V).to(torch.int32), "tokens": (flat % V).to(torch.int32)}


def _reorder(s):
    L, B, W, H, S, D = s["cache"].shape
    moved = s["cache"][:, torch.arange(B, device="cuda")[:, None], s["parents"].long()]
    live = torch.arange(S, device="cuda") < s["lens"][:, None]
    s["cache"].copy_(torch.where(live[None, :, None, None, :, None], moved, s["cache"]))
    return s["cache"]


def _context():
    """The handle that a program creates once."""
    global _handle
    from paper_2405_19715_b200 import specdec
    if _handle is None:
        _handle = specdec.Context(1, 1)
    return specdec, _handle


def run(state):
    s = state
    op = s["op"]
    if own:
        sd, ctx = _context()
        if op == "record":
            values, tokens, lse = sd.specdec_top_logits(ctx, s["logits"], s["k"], s["T"])
            return {"values": values, "tokens": tokens, "lse": lse}
        if op == "step":
            loss, grad = sd.specdec_distill_step(ctx, s["logits"], s["values"], s["tokens"], s["lse"], s["weight"], s["T"])
            return {"loss": loss, "grad": grad}
        if op == "pair":
            loss, saved = sd.specdec_distill(ctx, s["logits"], s["values"], s["tokens"], s["lse"], s["T"])
            grad = sd.specdec_distill_backward(ctx, s["logits"], s["values"], s["tokens"], s["lse"], saved, s["weight"], s["T"])
            return {"loss": loss, "grad": grad}
        if op == "beam":
            scores, parents, tokens = sd.specdec_beam_select(ctx, s["logits"], s["scores"], s["M"], s["T"], finished=s["finished"], end_token=0)
            return {"scores": scores, "parents": parents, "tokens": tokens}
        sd.specdec_beam_reorder(ctx, s["parents"], s["cache"], batch_dim=1, step_dim=4, lens=s["lens"])
        return s["cache"]
    if op == "record":
        return _record(s)
    if op in ("step", "pair"):
        loss, kept = _distill(s)
        return {"loss": loss, "grad": _gradient(s, kept, s["weight"])}
    return _beam(s) if op == "beam" else _reorder(s)


def work(case):
    c, es = case, _SIZE[case["dtype"]]
    if c["op"] == "reorder":
        # half to the full length; a beam is moved unless it is its own parent, a parent is read once however many follow it
        W, steps = c["W"], (max(1, c["longest"] // 2) + c["longest"]) / 2
        one = c["L"] * c["B"] * c["H"] * steps * c["D"] * es
        return {"bytes": one * (W * (1 - 1 / W) + W * (1 - (1 - 1 / W) ** (W - 1))), "flops": 0}
    if c["op"] == "beam":
        n = c["B"] * c["W"] * c["V"]
        return {"bytes": n * es + c["B"] * (8 * c["W"] + 12 * c["M"]), "flops": 3 * n}
    n, record = c["rows"] * c["V"], 8 * c["rows"] * c["k"]
    live = 0.8 if c.get("padded") else 1.0
    if c["op"] == "record":
        return {"bytes": n * es + record + 4 * c["rows"], "flops": 3 * n}
    # a step reads the logits and writes their gradient; loss and gradient apart read them twice
    return {"bytes": n * es * ((1 if c["op"] == "step" else 2) * live + 1) + record + 12 * c["rows"], "flops": 6 * n}


# ------------------------------------------------------------------------------------------------ 64 bits


def exact(case, seed):
    """The operators' definitions in 64 bits, row block by row block."""
    s = prepare(case, seed)
    op, T = s["op"], s["T"] if "T" in s else 1.0
    if op == "reorder":
        return None  # moves what is there: nothing is computed
    if op == "beam":
        B, W, V = s["logits"].shape
        scores = []
        for b in range(B):
            lp = torch.log_softmax(s["logits"][b].double() / T, dim=1) + s["scores"][b].double()[:, None]
            if s["finished"] is not None:
                for w in torch.nonzero(s["finished"][b]).flatten().tolist():
                    lp[w] = float("-inf")
                    lp[w, 0] = s["scores"][b, w].double()
            scores.append(torch.topk(lp.flatten(), s["M"]).values)
        return {"scores": torch.stack(scores), "parents": None, "tokens": None}
    n, V = s["logits"].shape
    step = max(1, (1 << 26) // V)
    if op == "record":
        values, lse = [], []
        for at in range(0, n, step):
            x = s["logits"][at:at + step].double()
            values.append(torch.topk(x, s["k"], dim=1).values)
            lse.append(torch.logsumexp(x / T, dim=1))
        return {"values": torch.cat(values), "tokens": None, "lse": torch.cat(lse)}
    loss, grad = [], torch.zeros(n, V, dtype=torch.float64, device="cuda")
    for at in range(0, n, step):
        log_q = torch.log_softmax(s["logits"][at:at + step].double() / T, dim=1)
        tokens, values = s["tokens"][at:at + step].long(), s["values"][at:at + step].double() / T
        live = tokens[:, 0] >= 0
        where = tokens.clamp(min=0)
        log_p = values - (s["lse"][at:at + step].double()[:, None] if s["rest"] else torch.logsumexp(values, dim=1, keepdim=True))
        inside = torch.zeros_like(log_q, dtype=torch.bool).scatter_(1, where, True)
        each = (log_p.exp() * (log_p - log_q.gather(1, where))).sum(1)
        target = torch.zeros_like(log_q).scatter_(1, where, log_p.exp())
        mass = log_p.exp().sum(1)
        if s["rest"] and s["k"] < V:
            left = (1 - mass).clamp(min=0)
            log_rest = torch.logsumexp(log_q.masked_fill(inside, float("-inf")), dim=1)
            each = each + torch.where(left > 0, left * (left.log() - log_rest), 0.0)
            mass = mass + left
            target += (log_q - log_rest[:, None]).exp().masked_fill(inside, 0.0) * left[:, None]
        loss.append(torch.where(live, each, 0.0))
        w = torch.where(live, s["weight"][at:at + step].double() / T, 0.0)
        grad[at:at + step] = (log_q.exp() * mass[:, None] - target) * w[:, None]
    return {"loss": torch.cat(loss), "grad": grad}
