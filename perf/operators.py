"""Timed workloads of the operators beside the phrase boost: what programs ask about rows of logits and the tokens on them.

A recogniser's rows [rows, V] reach the tree as log-probs; around that its user wants to know how sure the model was of
the tokens a decoder emitted (log-probs, entropy, the alternatives), trains on the hypotheses a search found (the
gradient of those), and trains a student on the alternatives kept of a teacher.  Rows come from small heads (a thousand
tokens and the blank, so contiguous rows are odd) to the large vocabularies of multilingual and language models, in
three types, now and then padded to a round stride, with tokens masked to -inf (a constrained search) and rows whose
mask leaves nothing.
"""
import math

import torch

own = False  # whether run() makes the framework's calls, or computes the same in elementary operations

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    base = dict(pad=0, temp=1.0)
    lp = dict(base, op="logprobs", tokens=1, top=0, entropy=True, stats=False, masked=0.0)
    back = dict(base, op="backward", tokens=1, entropy=True, masked=0.0)
    learn = dict(base, op="distill", tail=False, ragged=False)
    return [
        # The smallest call: confidence of the tokens a greedy step has just emitted, 32 hypotheses.
        dict(lp, name="logprobs_step", type="f32", rows=32, V=1024),
        # After a beam step of 32 utterances x 4 beams: tokens and 8 alternatives, head with a blank.
        dict(lp, name="logprobs_beam", type="f32", rows=128, V=1025, top=8),
        # One sequence of a large language model's vocabulary, single token, 20 alternatives.
        dict(lp, name="logprobs_one", type="bf16", rows=1, V=131072, top=20),
        # A serving step of 64 sequences over a multilingual vocabulary, a constrained search, 5 alternatives.
        dict(lp, name="logprobs_serve", type="f16", rows=64, V=50000, top=5, masked=0.9, temp=0.7),
        # All frames of 32 utterances, odd rows: frame confidences and 5 alternatives.
        dict(lp, name="logprobs_frames", type="f32", rows=16000, V=1025, top=5),
        # A teacher's pass: 32 alternatives a row are kept, at temperature 2.
        dict(lp, name="logprobs_teacher", type="bf16", rows=8192, V=32001, tokens=0, top=32, entropy=False, temp=2.0),
        # A training forward that scores 16 candidates a row (another model's alternatives), keeping what the gradient needs.
        dict(lp, name="logprobs_rescore", type="f16", rows=4096, V=8192, tokens=16, stats=True),
        # Gradient on the hypotheses of a small batch, odd rows, entropy bonus.
        dict(back, name="backward_frames", type="f32", rows=2000, V=1025),
        # The same over a multilingual vocabulary in training.
        dict(back, name="backward_large", type="bf16", rows=4096, V=50000),
        # A student's small batch: 8 entries a row, some rows shorter or padded.
        dict(learn, name="distill_frames", type="f32", rows=500, V=1025, K=8, ragged=True),
        # Few long rows: 64 tokens of a language model's vocabulary, 64 entries.
        dict(learn, name="distill_long", type="bf16", rows=64, V=131072, K=64, tail=True),
        # The largest: a training batch over 32000 tokens and the blank, 32 entries and the rest of the mass.
        dict(learn, name="distill_batch", type="bf16", rows=8192, V=32001, K=32, tail=True, temp=2.0),
    ]


MOST_CELLS = 8192 * 32001


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "backward", "distill", "distill"])
    V = _log_int(rng, 128, 131072)
    shape = rng.random()
    if shape < 0.35:
        V = max(128, V // 64 * 64)          # a tokenizer's round size ...
    elif shape < 0.7:
        V = max(128, V // 64 * 64) + 1      # ... and with the blank
    c = dict(op=op, type=rng.choice(["f32", "f16", "bf16"]), V=V, temp=rng.choice([0.7, 1.0, 1.0, 2.0]))
    c["pad"] = -V % 64 if rng.random() < 0.3 else 0
    most = MOST_CELLS // (2 if c["type"] == "f32" else 1) // (V + c["pad"])
    c["rows"] = max(1, min(_log_int(rng, 1, 16384), most))
    if op == "distill":
        c["K"] = _log_int(rng, 1, 64)
        c["tail"], c["ragged"] = rng.random() < 0.5, rng.random() < 0.3
    else:
        c["tokens"] = rng.choice([1, 1, 1, _log_int(rng, 2, 64)])
        c["entropy"] = rng.random() < 0.6
        c["masked"] = rng.choice([0.0, 0.0, 0.5, 0.95])
    if op == "logprobs":
        c["top"] = rng.choice([0, 1, 5, _log_int(rng, 2, 64)])
        c["stats"] = rng.random() < 0.3
        if c["top"]:
            c["tokens"] = rng.choice([0, c["tokens"]])
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------

def _gen(seed, k):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + k)
    return g


def _slices(c):
    step = max(1, (1 << 26) // c["V"])
    return [slice(i, min(c["rows"], i + step)) for i in range(0, c["rows"], step)]


def _scale(c):
    """Weight of a row: its share of the batch, or, where gradients are kept in fp16, a loss scale."""
    return 256.0 if c["type"] == "f16" else 1.0 / c["rows"]


def _inputs(c, seed):
    """Logits as a head leaves them: tails as long as those of trained models (the probabilities of the first tokens fall
    like a power of their rank), in six rows of ten one token further ahead; masked to -inf at random, one row in 97 of a
    masked batch as a whole."""
    rows, V, kind = c["rows"], c["V"], TYPES[c["type"]]
    g = _gen(seed, 1)
    held = torch.zeros((rows, V + c["pad"]), dtype=kind, device=DEV)
    d = {"case": c, "logits": held[:, :V]}
    if c["op"] == "distill":
        d["teacher_tokens"] = torch.empty((rows, c["K"]), dtype=torch.int32, device=DEV)
        d["teacher_logp"] = torch.empty((rows, c["K"]), device=DEV)
    for s in _slices(c):
        n = s.stop - s.start
        x = torch.randn((n, V), generator=g, device=DEV)
        x *= 2.5 * torch.randn((n, V), generator=g, device=DEV).abs()
        ahead = torch.randint(0, V, (n, 1), generator=g, device=DEV)
        x.scatter_add_(1, ahead, 8.0 * (torch.rand((n, 1), generator=g, device=DEV) < 0.6))
        if c["op"] == "distill":  # the student's row is the teacher's with noise
            best = torch.log_softmax(x / c["temp"], dim=1).topk(c["K"], dim=1)
            d["teacher_tokens"][s], d["teacher_logp"][s] = best.indices.to(torch.int32), best.values
            x = 0.8 * x + torch.randn((n, V), generator=g, device=DEV)
        elif c["masked"]:
            barred = torch.rand((n, V), generator=g, device=DEV) < c["masked"]
            barred |= (torch.arange(s.start, s.stop, device=DEV) % 97 == 41)[:, None]
            x.masked_fill_(barred, -math.inf)
        d["logits"][s] = x.to(kind)
    if c["op"] == "distill":
        if c["ragged"]:  # shorter lists, and rows behind the last frame: no entries
            size = torch.randint(0, c["K"] + 1, (rows, 1), generator=g, device=DEV)
            d["teacher_tokens"][torch.arange(c["K"], device=DEV)[None, :] >= size] = -1
        d["row_grads"] = torch.rand(rows, generator=g, device=DEV) * _scale(c)
    elif c["tokens"]:
        t = torch.randint(0, V, (rows, c["tokens"]), generator=g, device=DEV)
        sure = torch.rand(rows, generator=g, device=DEV) < 0.7
        t[:, 0] = torch.where(sure, d["logits"].argmax(dim=1), t[:, 0])
        d["tokens"] = t.to(torch.int32)
    if c["op"] == "backward":
        d["grad_logp"] = torch.randn((rows, c["tokens"]), generator=g, device=DEV) * _scale(c)
        d["grad_entropy"] = torch.full((rows,), -0.01 * _scale(c), device=DEV) if c["entropy"] else None
    return d


def prepare(c, seed):
    d = _inputs(c, seed)
    rows, V, kind = c["rows"], c["V"], TYPES[c["type"]]
    d["stream"] = int(torch.cuda.current_stream().cuda_stream)
    d["workspace"] = None
    if c["op"] == "logprobs":
        d["logp"] = torch.empty((rows, c["tokens"]), device=DEV) if c["tokens"] else None
        d["entropy"] = torch.empty(rows, device=DEV) if c["entropy"] else None
        d["top_tokens"] = torch.empty((rows, c["top"]), dtype=torch.int32, device=DEV) if c["top"] else None
        d["top_logp"] = torch.empty((rows, c["top"]), device=DEV) if c["top"] else None
        d["stats"] = torch.empty((rows, 3), device=DEV) if c["stats"] else None
    else:
        d["grad"] = torch.empty((rows, V), dtype=kind, device=DEV)
        d["loss"] = torch.empty(rows, device=DEV)
    if c["op"] == "backward":  # what the forward has left
        d["stats"] = torch.empty((rows, 3), device=DEV)
        for s in _slices(c):
            shifted, logsum, logp = _rows(d["logits"][s].float(), c["temp"])
            d["stats"][s] = torch.stack([d["logits"][s].float().amax(dim=1), logsum[:, 0], _entropy(logp)], dim=1)
    return d


# ---- one pass ------------------------------------------------------------------------------------------------------

def _rows(x, temp):
    """(x - max) / T, log of the sum of its exp, log-probs; a row that is -inf throughout: -inf, 0, -inf."""
    m = x.amax(dim=1, keepdim=True)
    shifted = (x - torch.where(m == -math.inf, torch.zeros_like(m), m)) / temp
    logsum = shifted.exp().sum(dim=1, keepdim=True).log()
    logsum = torch.where(m == -math.inf, torch.zeros_like(m), logsum)
    return shifted, logsum, shifted - logsum


def _entropy(logp):
    return -(logp.exp() * logp.clamp(min=-1e30)).sum(dim=1)


def _order(x):
    """Whole numbers in the order of (value descending, column ascending), largest first."""
    bits = (x + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64)
    return (key << 32) + torch.arange(x.shape[1] - 1, -1, -1, device=x.device)


def _dense(tokens, values, V):
    """values[r, k] added up at column tokens[r, k]; tokens outside the row are left out."""
    out = torch.zeros((tokens.shape[0], V + 1), dtype=values.dtype, device=values.device)
    return out.scatter_add_(1, torch.where(tokens >= 0, tokens.long(), V), values)[:, :V]


def _teacher(d):
    """The teacher's log-probs and probabilities, and what its list leaves of 1 (a small difference: in 64 bits; what fp32
    log-probs of whole rows may be off by, 2^-20, counts as nothing)."""
    there = d["teacher_tokens"] >= 0
    l = torch.where(there, d["teacher_logp"], -math.inf)
    if d["case"]["tail"]:
        rest = 1.0 - l.double().exp().sum(dim=1, keepdim=True)
        return l, l.exp(), torch.where(rest < 2.0 ** -20, torch.zeros_like(rest), rest).float()
    top = l.amax(dim=1, keepdim=True)
    e = (l - torch.where(top == -math.inf, torch.zeros_like(top), top)).exp()
    q = e / torch.where(top == -math.inf, torch.ones_like(top), e.sum(dim=1, keepdim=True))
    return torch.where(q > 0, q.log(), -math.inf), q, torch.zeros_like(top)


def _plain(d):
    c = d["case"]
    x = d["logits"].float()
    shifted, logsum, logp = _rows(x, c["temp"])
    if c["op"] == "logprobs":
        out = {}
        if c["tokens"]:
            out["logp"] = logp.gather(1, d["tokens"].long())
        if c["entropy"]:
            out["entropy"] = _entropy(logp)
        if c["stats"]:
            out["stats"] = torch.stack([x.amax(dim=1), logsum[:, 0], _entropy(logp)], dim=1)
        if c["top"]:
            first = c["V"] - 1 - (_order(x).topk(c["top"], dim=1).values & 0xFFFFFFFF)
            out["top_tokens"], out["top_logp"] = first.to(torch.int32), logp.gather(1, first)
        return out
    p = logp.exp()
    if c["op"] == "backward":
        grad = _dense(d["tokens"], d["grad_logp"], c["V"])
        pull = d["grad_logp"].sum(dim=1, keepdim=True)
        if c["entropy"]:
            pull = pull + d["grad_entropy"][:, None] * (logp.clamp(min=-1e30) + d["stats"][:, 2:])
        grad = torch.where(d["stats"][:, :1] == -math.inf, torch.zeros_like(p), (grad - p * pull) / c["temp"])
        return {"grad": grad.to(d["logits"].dtype)}
    log_q, q, q_rest = _teacher(d)
    at = d["teacher_tokens"].clamp(min=0).long()
    apart = log_q.double() - (shifted.gather(1, at) - logsum.double())  # (a small difference again)
    loss = torch.where(q > 0, q * apart, torch.zeros_like(apart)).sum(dim=1)
    mass = q.sum(dim=1, keepdim=True) + q_rest
    share = mass
    if c["tail"]:
        on_list = _dense(d["teacher_tokens"], torch.ones_like(q), c["V"]) > 0
        p_rest = torch.where(on_list, torch.zeros_like(p), p).sum(dim=1, keepdim=True)
        loss = loss + torch.where(q_rest > 0, q_rest * (q_rest / p_rest).double().log(), torch.zeros_like(q_rest).double())[:, 0]
        share = torch.where(on_list, mass, mass - q_rest / p_rest)
    grad = (p * share - _dense(d["teacher_tokens"], q, c["V"])) * (d["row_grads"][:, None] / c["temp"])
    return {"loss": loss.float(), "grad": grad.to(d["logits"].dtype)}


def run(d):
    if not own:
        return _plain(d)
    import paper_2508_07014_amd as pb
    c, x = d["case"], d["logits"]
    kind = {"f32": pb.PB_F32, "f16": pb.PB_F16, "bf16": pb.PB_BF16}[c["type"]]
    stride = c["V"] + c["pad"]
    if c["op"] == "backward":
        pb.pb_token_logprobs_backward(x, kind, stride, c["rows"], c["V"], c["temp"], d["stats"], d["tokens"], c["tokens"],
                                      d["grad_logp"], d["grad_entropy"], d["grad"], c["V"], d["stream"])
        return {"grad": d["grad"]}
    if d["workspace"] is None:
        size = (pb.pb_token_logprobs_workspace_bytes(kind, c["rows"], c["V"], c["top"]) if c["op"] == "logprobs" else
                pb.pb_distill_topk_workspace_bytes(kind, c["rows"], c["V"], c["K"]))
        d["workspace"] = torch.empty(max(16, size), dtype=torch.uint8, device=DEV)
    ws = d["workspace"]
    if c["op"] == "distill":
        mode = pb.PB_DISTILL_TAIL if c["tail"] else pb.PB_DISTILL_RENORM
        pb.pb_distill_topk(x, kind, stride, c["rows"], c["V"], c["temp"], d["teacher_tokens"], d["teacher_logp"], c["K"], mode,
                           d["row_grads"], d["loss"], d["grad"], c["V"], ws, ws.numel(), d["stream"])
        return {"loss": d["loss"], "grad": d["grad"]}
    pb.pb_token_logprobs(x, kind, stride, c["rows"], c["V"], c["temp"], d.get("tokens"), c["tokens"], c["top"], d["logp"],
                         d["entropy"], d["top_tokens"], d["top_logp"], d["stats"], ws, ws.numel(), d["stream"])
    return {k: d[k] for k in ("logp", "entropy", "stats", "top_tokens", "top_logp") if d[k] is not None}


def work(c):
    """Logits read once, every output written once; a subtraction, a product, an exponential and a sum a cell, and what the
    entropy, the gradient and the order of the alternatives need on top."""
    size = 4 if c["type"] == "f32" else 2
    rows, cells = float(c["rows"]), float(c["rows"]) * c["V"]
    if c["op"] == "logprobs":
        out = 8.0 * c["tokens"] + 8.0 * c["top"] + 4.0 * c["entropy"] + 12.0 * c["stats"]
        return {"bytes": cells * size + rows * out, "flops": cells * (4.0 + 2.0 * bool(c["entropy"] or c["stats"]) + bool(c["top"]))}
    if c["op"] == "backward":
        return {"bytes": 2.0 * cells * size + rows * (8.0 * c["tokens"] + 12.0 + 4.0 * c["entropy"]),
                "flops": cells * (5.0 + 2.0 * c["entropy"])}
    return {"bytes": 2.0 * cells * size + rows * (8.0 * c["K"] + 8.0), "flops": cells * (8.0 + c["tail"])}


# ---- the same in 64 bits, from the definition ----------------------------------------------------------------------

def _exact_rows(c, d, s):
    z = d["logits"][s].double() / c["temp"]
    V = c["V"]
    empty = (z == -math.inf).all(dim=1, keepdim=True)
    lse = torch.logsumexp(z, dim=1, keepdim=True)
    lp = torch.where(empty, torch.full_like(z, -math.inf), z - lse)
    p = lp.exp()
    H = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(dim=1)
    if c["op"] == "logprobs":
        top = d["logits"][s].double().amax(dim=1)
        r = {"logp": lp.gather(1, d["tokens"][s].long()) if c["tokens"] else None, "entropy": H if c["entropy"] else None}
        r["stats"] = torch.stack([top, torch.where(empty, torch.zeros_like(lse), lse - z.amax(dim=1, keepdim=True))[:, 0], H], dim=1)
        r["top_logp"] = lp.topk(c["top"], dim=1).values if c["top"] else None
        return r
    if c["op"] == "backward":
        dz = torch.zeros_like(z).scatter_add_(1, d["tokens"][s].long(), d["grad_logp"][s].double())
        dz -= p * d["grad_logp"][s].double().sum(dim=1, keepdim=True)
        if c["entropy"]:
            dz -= d["grad_entropy"][s].double()[:, None] * torch.where(p > 0, p * (lp + H[:, None]), torch.zeros_like(p))
        return {"grad": torch.where(empty, torch.zeros_like(dz), dz / c["temp"])}
    tok, l = d["teacher_tokens"][s].long(), d["teacher_logp"][s].double()
    l = l.masked_fill(tok < 0, -math.inf)
    some = (tok >= 0).any(dim=1, keepdim=True)
    if c["tail"]:
        rest = 1.0 - l.exp().sum(dim=1, keepdim=True)
        rest = rest.masked_fill(rest < 2.0 ** -20, 0.0)
    else:
        l = torch.where(some, l - torch.logsumexp(l, dim=1, keepdim=True), l)
        rest = torch.zeros_like(lse)
    q = l.exp()
    target = torch.zeros((len(z), V + 1), dtype=torch.float64, device=DEV)
    target.scatter_add_(1, tok.masked_fill(tok < 0, V), q)
    listed_too = torch.zeros_like(target, dtype=torch.bool).scatter_(1, tok.masked_fill(tok < 0, V), True)[:, :V]
    loss = torch.where(q > 0, q * (l - lp.gather(1, tok.clamp(min=0))), torch.zeros_like(q)).sum(dim=1)
    dz = p * (q.sum(dim=1, keepdim=True) + rest) - target[:, :V]
    if c["tail"]:
        p_rest = p.masked_fill(listed_too, 0.0).sum(dim=1, keepdim=True)
        loss += torch.where(rest > 0, rest * (rest.log() - p_rest.log()), torch.zeros_like(rest))[:, 0]
        dz -= p.masked_fill(listed_too, 0.0) * torch.where(rest > 0, rest / p_rest, torch.zeros_like(rest))
    return {"loss": loss, "grad": dz * (d["row_grads"][s].double()[:, None] / c["temp"])}


def exact(c, seed):
    d = _inputs(c, seed)
    parts = [_exact_rows(c, d, s) for s in _slices(c)]
    out = {k: torch.cat([p[k] for p in parts]) for k, v in parts[0].items() if v is not None}
    if c["op"] == "logprobs":
        out = {k: v for k, v in out.items() if k != "stats" or c["stats"]}
        if c["top"]:
            out["top_tokens"] = None
    return out
