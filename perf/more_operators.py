"""The answers of the softmax that the training of rows works with, and learning from another model's answers.

rnnd_contrast trains rows so that the softmax over minus squared distances puts a query's key first.  Two calls stand beside it:

- log probabilities: how probable a given key is for a query among all keys, how sure the model is (the entropy), and which
  keys are the most probable ones, exactly and in order (the graph's search is approximate, and gives no probabilities);
- distillation: a small model with short rows learns from a larger one, of which a query's most probable keys and their log
  probabilities are kept (what the first call gives).  The loss is the divergence of the student's softmax over all keys from
  the teacher's list, either renormalised or with the rest of the probability as one more outcome.

Shapes are those of this repository's own data: rows of 32, 96, 100, 768 coordinates, tables of up to 1,000,000 rows, batches
of up to 8,192 queries with 16,384 keys.  `run` computes the plain form in elementary torch operations where `own` is
false, and calls the library where it is true.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _logprob(name, B, M, d, rows, top, target=True):
    return {"name": name, "op": "logprob", "B": B, "M": M, "d": d, "rows": rows, "top": top, "target": target}


def _distill(name, B, M, d, rows, top, tail, grads=True):
    return {"name": name, "op": "distill", "B": B, "M": M, "d": d, "rows": rows, "top": top, "tail": tail, "grads": grads}


def listed():
    return [
        # one query answered from a small table, ten alternatives: latency
        _logprob("logprob_f32_1_20k_96", 1, 20_000, 96, "f32", 10, target=False),
        # one query answered from the whole of the largest table
        _logprob("logprob_f32_1_1m_96", 1, 1_000_000, 96, "f32", 10, target=False),
        # a few queries that arrive together, against a table of passages
        _logprob("logprob_bf16_4_300k_768", 4, 300_000, 768, "bf16", 20),
        # the held-out queries of a table of passages, every passage an alternative
        _logprob("logprob_bf16_200_300k_768", 200, 300_000, 768, "bf16", 20),
        # word vectors in float32: how good they are after an epoch
        _logprob("logprob_f32_2k_10k_100", 2_000, 10_000, 100, "f32", 10),
        # perplexity and entropy alone, half precision
        _logprob("logprob_f16_1k_11k_768", 1_000, 11_000, 768, "f16", 0),
        # the teacher's pass over a big batch: the 32 best keys of every query are what the student learns from
        _logprob("logprob_bf16_8k_16k_768", 8_192, 16_384, 768, "bf16", 32),
        # a small student in a small batch
        _distill("distill_f32_100_32", 100, 1_100, 32, "f32", 10, True),
        # word vectors of 100 coordinates learn from longer ones
        _distill("distill_f32_2k_100", 2_000, 10_000, 100, "f32", 10, True),
        # passages scored by a slower model: its scores of the 32 candidates, renormalised
        _distill("distill_bf16_1k_768", 1_000, 11_000, 768, "bf16", 32, False),
        # the loss alone, on held-out data
        _distill("distill_f16_loss_1k_768", 1_000, 11_000, 768, "f16", 32, True, grads=False),
        # the largest: a big batch against the teacher's 32 best keys and the rest
        _distill("distill_bf16_8k_768", 8_192, 16_384, 768, "bf16", 32, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    rows = rng.choice(["f32", "f16", "bf16"])
    d = min(768, rng.choice([_log_int(rng, 16, 960), 16 * _log_int(rng, 1, 60)]))
    room = 8_192 * 16_384 * 768 // (6 if rows == "f32" else 1)      # single precision costs several times as much
    top = _log_int(rng, 1, 64)
    if rng.random() < 0.5:
        few = rng.random() < 0.4
        M = _log_int(rng, 150, min(1_000_000, 230_400_000 // d))
        B = rng.randint(1, 8) if few else _log_int(rng, 1, 8_192)
        B = max(1, min(B, 134_217_728 // M, room // (M * d)))
        return {"op": "logprob", "B": B, "M": M, "d": d, "rows": rows, "top": rng.choice([0, top, top]), "target": rng.random() < 0.7}
    B = _log_int(rng, 1, 8_192)
    M = max(200, min(16_384, B * rng.randint(1, 12) + rng.randint(0, 300)))
    if rows == "f32":
        B, M = min(B, 3_000), min(M, 12_000)
    return {"op": "distill", "B": B, "M": M, "d": d, "rows": rows, "top": top, "tail": rng.random() < 0.6, "grads": rng.random() < 0.8}


# ---------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + len(case["op"]))
    B, M, d, k, t = case["B"], case["M"], case["d"], case["top"], TYPES[case["rows"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    def share(n, p):
        return torch.rand(n, device="cuda", generator=g) < p

    def unit(x):
        return x / x.norm(dim=1, keepdim=True)

    s = {"case": case, "scale": 5.0}
    topics = min(64, 1 + M // 16)
    keys = normal(topics, d)[torch.randint(0, topics, (M,), device="cuda", generator=g)]
    keys += 0.7 * normal(M, d)
    keys = unit(keys)
    order = torch.randperm(M, device="cuda", generator=g)
    order = order[:B] if B <= M else order.repeat(-(-B // M))[:B]
    q = unit(keys[order] + normal(B, d) / math.sqrt(d))
    s["key_ids"] = torch.randperm(M, device="cuda", generator=g).to(torch.int32)
    s["query_ids"] = torch.full((B,), M, device="cuda", dtype=torch.int32)
    itself = share(B, 0.3)                                      # queries that are rows of the table: never their own answer
    s["query_ids"][itself] = s["key_ids"][order[itself]]
    gone = share(M, 0.01)                                       # rows taken out of the table
    s["bias"] = -2.0 * torch.rand(M, device="cuda", generator=g)     # log of how often a row is asked for
    if case["op"] == "logprob":
        if case["target"]:
            s["target"] = torch.where(itself, torch.randint(0, M, (B,), device="cuda", generator=g), order).to(torch.int32)
            s["target"][share(B, 0.01)] = -1
    else:
        # the teacher's rows are others: near the student's in what they say
        theirs = unit(keys + 0.5 * normal(M, d) / math.sqrt(d))
        logits = 16.0 * (unit(q + 0.5 * normal(B, d) / math.sqrt(d)) @ theirs.T)
        logits[:, gone] = -math.inf
        logits.masked_fill_(s["key_ids"][None, :] == s["query_ids"][:, None], -math.inf)
        best, at = logits.topk(k, dim=1)
        s["teacher_logits"] = best - torch.logsumexp(logits, 1, keepdim=True) if case["tail"] else best.clone()
        s["teacher_ids"] = at.to(torch.int32)
        short = share(B, 0.1)                                   # queries for which the teacher kept fewer
        s["teacher_ids"][short, (k + 1) // 2:] = -1
        s["teacher_ids"][share(B, 0.01)] = -1                   # ... or none
        s["weight"] = (0.5 + torch.rand(B, device="cuda", generator=g)) * ((1024.0 if case["rows"] == "f16" else 1.0) / B)
    s["key_ids"][gone] = -1
    s["Q"], s["K"] = q.to(t), keys.to(t)
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _logits(s):
    """Logits, but for -scale |q|^2, which is the same in a whole row; -inf where a key is left out."""
    q, k = s["Q"].float(), s["K"].float()
    gone = s["key_ids"] < 0
    logits = torch.addmm((s["bias"] - s["scale"] * k.square().sum(1))[None, :], q, k.T, alpha=2 * s["scale"])
    return logits.masked_fill_((s["key_ids"][None, :] == s["query_ids"][:, None]) | gone[None, :], -math.inf)


def _softmax_sums(logits):
    top = logits.amax(1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    below = logits - top
    e = torch.exp(below)
    return top, below, e, e.sum(1, keepdim=True)


def _run_logprob(s):
    case, M, k = s["case"], s["case"]["M"], s["case"]["top"]
    logits = _logits(s)
    top, below, e, total = _softmax_sums(logits)
    log_total = torch.log(total)
    got = {"entropy": log_total[:, 0] - torch.where(e > 0, e * below, 0.0).sum(1) / total[:, 0]}
    if case["target"]:
        target = s["target"].long()
        at = target.clamp(0, M - 1)[:, None]
        mine = logits.gather(1, at)
        valid = ((target >= 0) & (target < M))[:, None] & (mine > -math.inf)
        got["logprob"] = torch.where(valid, (mine - top) - log_total, 0.0)[:, 0]
    if k:
        # the order of neighbours is decided in double precision, for a few more than are asked for
        best, at = logits.topk(min(M, k + 8), dim=1)
        at, order = at.sort(1)
        best = best.gather(1, order)
        exactly = torch.empty(at.shape, device="cuda", dtype=torch.float64)
        step = max(1, 100_000_000 // (at.shape[1] * case["d"]))
        for i in range(0, len(at), step):
            rows = s["K"][at[i:i + step]].double()
            both = (rows * (2.0 * s["Q"][i:i + step].double()[:, None, :] - rows)).sum(2)
            exactly[i:i + step] = s["bias"].double()[at[i:i + step]] + s["scale"] * both
        exactly.masked_fill_(best == -math.inf, -math.inf)
        exactly, order = exactly.sort(dim=1, descending=True, stable=True)
        exactly, order = exactly[:, :k], order[:, :k]
        got["top_ids"] = torch.where(exactly > -math.inf, at.gather(1, order), -1).to(torch.int32)
        got["top_logprob"] = (exactly - top - log_total).float()
    return got


def _list(s):
    """Which entries of the teachers' lists count, and their keys."""
    ids, M = s["teacher_ids"].long(), s["case"]["M"]
    at = ids.clamp(0, M - 1)
    on = (ids >= 0) & (ids < M) & (s["teacher_logits"] > -math.inf)
    name = s["key_ids"][at]
    on &= (name >= 0) & (name != s["query_ids"][:, None])
    again = (ids[:, :, None] == ids[:, None, :]) & on[:, None, :]       # named before
    return at, on & ~again.tril(-1).any(2)


def _run_distill(s):
    case = s["case"]
    logits = _logits(s)
    at, on = _list(s)
    counts = on.any(1)[:, None]
    mine = logits.gather(1, at)
    listed_keys = torch.zeros_like(logits, dtype=torch.bool)
    row = torch.arange(len(at), device="cuda")[:, None].expand_as(at)
    listed_keys[row[on], at[on]] = True
    top, _, e, total = _softmax_sums(logits)
    lse = top + torch.log(total)
    off = torch.where(listed_keys, 0.0, e).sum(1, keepdim=True)      # the student's mass off the list, over exp(top)
    wide = s["teacher_logits"].double().masked_fill(~on, -math.inf)
    if case["tail"]:
        p = wide.exp()
        rest = torch.where(off > 0, (1.0 - p.sum(1, keepdim=True)).clamp(min=0.0), 0.0)
    else:
        p = (wide - torch.where(counts, wide.amax(1, keepdim=True), 0.0)).exp()
        rest = torch.zeros_like(p[:, :1])
    mass = torch.where(counts, p.sum(1, keepdim=True) + rest, 1.0)
    p, rest = (p / mass).float(), (rest / mass).float()
    each = torch.where(p > 0, p * (torch.log(p) - (mine - lse)), 0.0).sum(1, keepdim=True)
    tail = torch.where(rest > 0, rest * (torch.log(rest) - torch.log(off / total)), 0.0)
    loss = torch.where(counts, each + tail, 0.0)[:, 0]
    if not case["grads"]:
        return {"loss": loss}
    q = torch.where(counts, s["Q"].float(), 0.0)
    k = torch.where((s["key_ids"] < 0)[:, None], 0.0, s["K"].float())
    prob = e / total
    g = torch.where(listed_keys, prob, prob * (1.0 - torch.where(rest > 0, rest / (off / total), 0.0)))
    g.scatter_add_(1, at, -torch.where(on, p, 0.0))
    g = torch.where(counts, g * s["weight"][:, None], 0.0)
    dq = 2 * s["scale"] * (g @ k)
    dk = 2 * s["scale"] * (g.T @ q - g.sum(0)[:, None] * k)
    return {"loss": loss, "dq": dq.to(s["Q"].dtype), "dk": dk.to(s["K"].dtype)}


def run(s):
    if own:
        return _run_own(s)
    return _run_logprob(s) if s["case"]["op"] == "logprob" else _run_distill(s)


def _run_own(s):
    import paper_2310_20419_amd as rn
    case = s["case"]
    if case["op"] == "logprob":
        logprob, entropy, ids, top = rn.rnnd_logprob(s["Q"], s["K"], s["scale"], target=s.get("target"), alternatives=case["top"],
                                                     query_ids=s["query_ids"], key_ids=s["key_ids"], key_bias=s["bias"])
        got = {"entropy": entropy}
        if case["target"]:
            got["logprob"] = logprob
        if case["top"]:
            got["top_ids"], got["top_logprob"] = ids, top
        return got
    loss, dq, dk = rn.rnnd_distill(s["Q"], s["K"], s["teacher_ids"], s["teacher_logits"], s["scale"], tail=case["tail"],
                                   query_ids=s["query_ids"], key_ids=s["key_ids"], key_bias=s["bias"], row_weight=s["weight"],
                                   want_grad=case["grads"])
    return {"loss": loss, "dq": dq, "dk": dk} if case["grads"] else {"loss": loss}


# ---------------------------------------------------------------------------------------------------- work, 64 bits
def work(case):
    B, M, d, k = case["B"], case["M"], case["d"], case["top"]
    rows = (B + M) * d * SIZE[case["rows"]]
    if case["op"] == "logprob":
        return {"bytes": rows + 8 * M + 4 * B + (8 if case["target"] else 0) * B + 4 * B + 8 * B * k, "flops": 2 * B * M * d}
    return {"bytes": rows * (2 if case["grads"] else 1) + 8 * M + 12 * B + 8 * B * k, "flops": 2 * B * M * d * (3 if case["grads"] else 1)}


def exact(case, seed):
    """The definitions in double precision."""
    s = prepare(case, seed)
    B, M = case["B"], case["M"]
    q, k = s["Q"].double(), s["K"].double()
    if case["op"] == "distill" and case["grads"]:
        q.requires_grad_()
        k.requires_grad_()
    far = q.square().sum(1)[:, None] + (k.square().sum(1)[None, :] - 2 * (q @ k.T))
    names = s["key_ids"]
    out = (names < 0)[None, :] | (names[None, :] == s["query_ids"][:, None])
    logits = (s["bias"].double()[None, :] - s["scale"] * far).masked_fill(out, -math.inf)
    logs = torch.log_softmax(logits, 1)
    if case["op"] == "logprob":
        got = {"entropy": -torch.where(out, 0.0, logs.exp() * logs.masked_fill(out, 0.0)).sum(1)}
        if case["target"]:
            target = s["target"].long()
            asked = target >= 0
            p = logs[asked, target[asked]]
            got["logprob"] = torch.zeros(B, device="cuda", dtype=torch.float64)
            got["logprob"][asked] = torch.where(p > -math.inf, p, 0.0)
        if case["top"]:
            if B * M <= 16_000_000 or M <= 20_000:
                best, at = logs.sort(dim=1, descending=True, stable=True)
            else:       # long rows, a few at a time
                parts = [row.sort(descending=True, stable=True) for row in logs]
                best, at = (torch.stack([x[:case["top"]] for x in both]) for both in zip(*parts))
            got["top_ids"], got["top_logprob"] = at[:, :case["top"]].to(torch.int32), best[:, :case["top"]]
        return got
    # every query's distribution over all keys and, with the tail, the keys off its list taken together
    ids = s["teacher_ids"].long()
    p = torch.zeros(B, M + 1, device="cuda", dtype=torch.float64)
    for t in range(case["top"]):
        row = (ids[:, t] >= 0).nonzero()[:, 0]
        row = row[~out[row, ids[row, t]]]
        fresh = p[row, ids[row, t]] == 0
        p[row[fresh], ids[row[fresh], t]] = s["teacher_logits"].double()[row[fresh], t].exp()
    counts = (p > 0).any(1)
    if case["tail"]:
        p[:, M] = (1 - p.sum(1)).clamp(min=0)
    p = p[counts] / p[counts].sum(1, keepdim=True)
    mine, on = logs[counts], p[:, :M] > 0
    loss = torch.zeros(B, device="cuda", dtype=torch.float64)
    each = (torch.special.xlogy(p[:, :M], p[:, :M]) - p[:, :M] * mine.masked_fill(~on, 0.0)).sum(1)
    if case["tail"]:
        off = torch.logsumexp(mine.masked_fill(on, -math.inf), 1)
        each = each + torch.special.xlogy(p[:, M], p[:, M]) - p[:, M] * off
    loss[counts] = each.detach()
    if not case["grads"]:
        return {"loss": loss}
    if not counts.any():
        return {"loss": loss, "dq": torch.zeros_like(q), "dk": torch.zeros_like(k)}
    dq, dk = torch.autograd.grad((s["weight"].double()[counts] * each).sum(), (q, k))
    return {"loss": loss, "dq": dq, "dk": dk}
