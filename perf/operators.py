"""Operators on rows of logits: how likely given tokens are, how uncertain a row is and which tokens come next in
line, the loss that pulls a student's rows towards a teacher's top logits, the gradients of both, and the output head
that gives the statistics without storing its logits.  ``run`` computes each in plain torch operations in 32 bits, or,
where ``own`` is true, through the library's calls.

For a row x of V logits at temperature tau, m = max x, L = ln sum_j exp((x_j - m) / tau), p_j = exp((x_j - m) / tau - L).
A row whose logits are all -inf has p = 0: its statistics are -inf, its entropy 0, its gradients 0."""
import math
import random

import torch

own = False
DEV = "cuda"


# ---------------------------------------------------------------------------------------------------------- cases
def _logprobs(name, rows, V, dtype, n_alt, entropy, tau=1.0, masked=False, pad=0):
    return {"name": name, "op": "logprobs", "rows": rows, "V": V, "dtype": dtype, "n_alt": n_alt, "entropy": entropy, "tau": tau, "masked": masked, "pad": pad}


def _logprobs_grad(name, rows, V, dtype, entropy, tau=1.0, masked=False, pad=0):
    return {"name": name, "op": "logprobs_grad", "rows": rows, "V": V, "dtype": dtype, "entropy": entropy, "tau": tau, "masked": masked, "pad": pad}


def _distill(name, rows, V, dtype, K, what, tau=1.0, masked=False, pad=0):
    return {"name": name, "op": "distill", "rows": rows, "V": V, "dtype": dtype, "K": K, "what": what, "tau": tau, "masked": masked, "pad": pad}


def _linear(name, rows, C, V, tau=1.0):
    return {"name": name, "op": "linear", "rows": rows, "C": C, "V": V, "tau": tau}


def listed():
    return [
        # the first scale of two images: one token each, answered while the next scale waits
        _logprobs("logprobs_first_scale", 2, 4096, "float32", 5, True),
        # every token of two 64 x 64 maps scored after the last scale, with what else the head would have taken
        _logprobs("logprobs_maps_64", 8192, 4096, "float32", 8, True),
        # single tokens of four sequences over a large vocabulary, 20 alternatives each
        _logprobs("logprobs_tokens_large_vocab", 4, 131072, "bfloat16", 20, True, tau=0.8),
        # a ragged batch over an odd vocabulary, some rows with most of their tokens forbidden, some with all
        _logprobs("logprobs_odd_vocab", 3001, 50021, "bfloat16", 20, True, tau=1.3, masked=True),
        # training on the tokens of two 64 x 64 maps with an entropy bonus
        _logprobs_grad("logprobs_grad_maps_64", 8192, 4096, "float32", True),
        # training over an odd vocabulary whose rows lie in a wider tensor
        _logprobs_grad("logprobs_grad_odd_vocab", 2003, 50021, "bfloat16", False, tau=0.9, masked=True, pad=27),
        # a pruned schedule's head pulled towards the unpruned one's on two 64 x 64 maps: loss and gradient in one call
        _distill("distill_maps_64", 8192, 4096, "float32", 16, "loss_and_grad", tau=2.0),
        # the largest: a training batch over a large vocabulary
        _distill("distill_large_vocab", 4096, 131072, "bfloat16", 64, "loss_and_grad"),
        # how far a pruned schedule's rows are from the unpruned one's, as a measure
        _distill("distill_measure", 1025, 32768, "bfloat16", 32, "loss", masked=True),
        # loss first, gradient when the weight of each row is known
        _distill("distill_loss_then_grad", 2048, 16384, "float32", 32, "loss_then_grad", tau=1.5),
        # the head over two 64 x 64 maps: likelihood of their tokens, no logits kept
        _linear("linear_maps_64", 8192, 2048, 4096),
        # the same for one 13 x 13 map of a smaller model
        _linear("linear_map_13", 169, 1024, 4096),
    ]


MOST_ELEMENTS = 256 << 20      # of one call; the largest listed case has 512 Mi


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "logprobs_grad", "distill", "distill", "linear"])
    tau = rng.choice([1.0, round(rng.uniform(0.5, 2.5), 3)])
    if op == "linear":
        c = _linear(None, _log_int(rng, 1, 8192), 64 * _log_int(rng, 2, 32), 8 * _log_int(rng, 32, 2048), tau)
    else:
        V = _log_int(rng, 200, 200000)
        rows = _log_int(rng, 1, max(1, min(16384, MOST_ELEMENTS // V)))
        dtype = rng.choice(["float32", "bfloat16"])
        masked, pad = rng.random() < 0.4, rng.choice([0, 0, rng.randint(1, 64)])
        if op == "logprobs":
            c = _logprobs(None, rows, V, dtype, rng.choice([0, 1, rng.randint(2, 32), rng.randint(2, 64)]), rng.random() < 0.7, tau, masked, pad)
        elif op == "logprobs_grad":
            c = _logprobs_grad(None, rows, V, dtype, rng.random() < 0.5, tau, masked, pad)
        else:
            c = _distill(None, rows, V, dtype, _log_int(rng, 1, 128), rng.choice(["loss", "loss_and_grad", "loss_then_grad"]), tau, masked, pad)
    del c["name"]
    return c


def work(case):
    rows, V = case["rows"], case["V"]
    if case["op"] == "linear":
        C = case["C"]
        return {"bytes": 2.0 * (rows * C + V * C + V) + 20.0 * rows, "flops": 2.0 * rows * V * C}
    es = 4.0 if case["dtype"] == "float32" else 2.0
    if case["op"] == "logprobs":
        return {"bytes": es * rows * V + rows * (4.0 + 12.0 + 4.0 * case["entropy"] + 8.0 * case["n_alt"]), "flops": 5.0 * rows * V}
    if case["op"] == "logprobs_grad":
        return {"bytes": 2 * es * rows * V + rows * (16.0 + 8.0 * case["entropy"]), "flops": 6.0 * rows * V}
    grad = case["what"] != "loss"
    return {"bytes": es * rows * V * (1 + grad) + rows * (8.0 * case["K"] + 12.0 + 4.0 * grad), "flops": (5.0 + 3.0 * grad) * rows * V}


# --------------------------------------------------------------------------------------------------------- inputs
def _inputs(case, seed):
    """Everything that a program has before the call, from the seed alone."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, device=DEV, generator=g)
    u = lambda *s: torch.rand(*s, device=DEV, generator=g)
    rows, V = case["rows"], case["V"]
    s = {}
    if case["op"] == "linear":
        C = case["C"]
        s["a"] = (n(rows, C)).bfloat16()                     # a layer-normalised row has unit variance
        s["w"] = (n(V, C) * (2.5 / math.sqrt(C))).bfloat16()
        s["b"] = (n(V) * 0.1).bfloat16()
        s["ids"] = (u(rows) * V).long().clamp_(max=V - 1).to(torch.int32)
        return s
    dtype = getattr(torch, case["dtype"])
    wide = n(rows, V + case["pad"]).mul_(2.5).add_(4.0 * n(rows, 1))
    # a few tokens that the row prefers, as a trained head has them
    wide.scatter_add_(1, (u(rows, 6) * V).long().clamp_(max=V - 1), 6.0 * u(rows, 6))
    teacher = wide[:, :V] + 0.7 * n(rows, V) if case["op"] == "distill" else None
    ids = (u(rows) * V).long().clamp_(max=V - 1)
    if case["op"] != "distill":                              # half of the given tokens are the row's own choice
        ids = torch.where(u(rows) < 0.5, wide[:, :V].argmax(1), ids)
    if case["masked"]:                                       # a quarter of the rows forbid most tokens, a few forbid all
        r = u(rows, 1)
        keep = torch.where(r < 0.25, 0.02 + 0.1 * r, torch.where(r > 0.98, torch.zeros_like(r), torch.ones_like(r)))
        wide.masked_fill_(u(rows, V + case["pad"]) >= keep, -math.inf)
    ids = torch.where(u(rows) < 0.05, torch.full_like(ids, -1), ids)     # padding: rows without a token
    s["logits"] = wide.to(dtype)[:, :V]
    if case["op"] == "distill":
        K = min(case["K"], V)
        top = teacher.topk(K, dim=1)
        t_ids, t_logits = top.indices.to(torch.int32), top.values
        t_ids = torch.where(u(rows, K) < 0.02, torch.full_like(t_ids, -1), t_ids)   # entries that the teacher's list lacks
        if case["masked"]:                                   # a teacher with the same forbidden tokens
            lost = torch.isinf(torch.gather(s["logits"].float(), 1, t_ids.long().clamp(min=0)))
            t_ids = torch.where(lost, torch.full_like(t_ids, -1), t_ids)
        s["t_ids"], s["t_logits"] = t_ids, t_logits
        s["g"] = (0.5 + u(rows)) / rows                      # weight of each row's loss
        return s
    s["ids"] = ids.to(torch.int32)
    if case["op"] == "logprobs_grad":
        s["g_logprob"] = -(0.5 + u(rows)) / rows
        s["g_entropy"] = 0.01 * (0.5 + u(rows)) / rows if case["entropy"] else None
        x = s["logits"].float()
        m = x.amax(1)
        m0 = torch.where(torch.isinf(m), torch.zeros_like(m), m)[:, None]
        d = (x - m0) / case["tau"]
        e = d.exp()
        L = e.sum(1).log()
        s["stats"] = torch.stack([m, L], 1)                  # what the forward call has left
        h = L - (e * d.clamp(min=-1e30)).sum(1) / e.sum(1)
        s["entropy"] = torch.where(torch.isinf(L), torch.zeros_like(h), h) if case["entropy"] else None
    return s


def prepare(case, seed):
    return dict(case, **_inputs(case, seed))


# ----------------------------------------------------------------------------------------------------- plain forms
def _statistics(x, tau):
    """(m, 0 in its place where the row is empty, (x - m) / tau, exp of that, its sum, L), kept as columns."""
    m = x.amax(1, keepdim=True)
    m0 = torch.where(m == -math.inf, torch.zeros_like(m), m)
    d = (x - m0) / tau
    e = d.exp()
    total = e.sum(1, keepdim=True)
    return m, d, e, total, total.log()


def _logprob_of(d, L, ids):
    lp = torch.gather(d, 1, ids.long().clamp(min=0)) - L
    return torch.where(ids < 0, torch.zeros_like(lp), torch.where(L == -math.inf, torch.full_like(lp, -math.inf), lp))


def _entropy(d, e, total, L):
    h = L - (e * d.clamp(min=-1e30)).sum(1, keepdim=True) / total
    return torch.where(L == -math.inf, torch.zeros_like(h), h)


def _alternatives(x, n_alt):
    """The n_alt largest of each row, ties to the lowest index: the value's bits in an order of integers, then the index."""
    V = x.shape[1]
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    key = (bits << 32) | (V - 1 - torch.arange(V, device=x.device))
    ids = V - 1 - (key.topk(n_alt, dim=1).values & 0xFFFFFFFF)
    return torch.where(torch.gather(x, 1, ids) == -math.inf, torch.full_like(ids, -1), ids)


def _plain_logprobs(s):
    x, ids = s["logits"].float(), s["ids"][:, None]
    m, d, e, total, L = _statistics(x, s["tau"])
    out = {"logprob": _logprob_of(d, L, ids)[:, 0], "stats": torch.cat([m, L], 1)}
    if s["entropy"]:
        out["entropy"] = _entropy(d, e, total, L)[:, 0]
    if s["n_alt"]:
        alt = _alternatives(x, s["n_alt"])
        lp = torch.gather(d, 1, alt.clamp(min=0)) - L
        out["alt_ids"] = alt.to(torch.int32)
        out["alt_logprob"] = torch.where(alt < 0, torch.full_like(lp, -math.inf), lp)
    return out


def _plain_logprobs_grad(s):
    x, ids, tau = s["logits"].float(), s["ids"][:, None].long(), s["tau"]
    m, L = s["stats"][:, :1], s["stats"][:, 1:]
    empty = L == -math.inf
    lp = (x - torch.where(empty, torch.zeros_like(m), m)) / tau - torch.where(empty, torch.zeros_like(L), L)
    p = lp.exp()
    g = torch.where(ids < 0, torch.zeros_like(L), s["g_logprob"][:, None])
    dx = -g * p
    if s["g_entropy"] is not None:
        dx = dx - s["g_entropy"][:, None] * p * (lp.clamp(min=-1e30) + s["entropy"][:, None])
    dx = dx.scatter_add(1, ids.clamp(min=0), torch.where(empty, torch.zeros_like(g), g))
    return (dx / tau).to(s["logits"].dtype)


def _plain_distill(s):
    x, tau, V = s["logits"].float(), s["tau"], s["V"]
    m, d, e, total, L = _statistics(x, tau)
    ids = s["t_ids"].long()
    t = torch.where(ids < 0, torch.full_like(s["t_logits"], -math.inf), s["t_logits"])
    _, td, te, ttotal, tL = _statistics(t, tau)
    q = torch.where(tL == -math.inf, torch.zeros_like(te), te / ttotal)
    logq = td - tL
    lp = torch.gather(d, 1, ids.clamp(min=0)) - L
    lp = torch.where(L == -math.inf, torch.full_like(lp, -math.inf), lp)
    out = {"loss": torch.where(q > 0, q * (logq - lp), torch.zeros_like(q)).sum(1), "stats": torch.cat([m, L], 1)}
    if s["what"] != "loss":
        empty = L == -math.inf
        p = torch.where(empty, torch.zeros_like(e), e / total)
        dx = p * (q.sum(1, keepdim=True) > 0)                       # a row without entries has no gradient
        dx = dx.scatter_add(1, ids.clamp(min=0), torch.where(empty, torch.zeros_like(q), -q))
        out["dlogits"] = (dx * (s["g"][:, None] / tau)).to(s["logits"].dtype)
    return out


def _plain_linear(s):
    x = s["a"].float() @ s["w"].float().t() + s["b"].float()
    m, d, e, total, L = _statistics(x, s["tau"])
    return {"logprob": _logprob_of(d, L, s["ids"][:, None])[:, 0], "stats": torch.cat([m, L], 1), "entropy": _entropy(d, e, total, L)[:, 0]}


def run(s):
    if own:
        return _own(s)
    return {"logprobs": _plain_logprobs, "logprobs_grad": _plain_logprobs_grad, "distill": _plain_distill, "linear": _plain_linear}[s["op"]](s)


def _own(s):
    from paper_2503_23367_b200 import binding as fv
    op = s["op"]
    if op == "logprobs":
        return fv.fv_token_logprobs(s["logits"], s["ids"], tau=s["tau"], n_alt=s["n_alt"], want_entropy=s["entropy"])
    if op == "logprobs_grad":
        return fv.fv_token_logprobs_grad(s["logits"], s["ids"], s["stats"], s["g_logprob"], tau=s["tau"], entropy=s["entropy"], g_entropy=s["g_entropy"])
    if op == "linear":
        return fv.fv_linear_logprobs(s["a"], s["w"], s["b"], s["ids"], tau=s["tau"], want_entropy=True)
    if s["what"] == "loss_and_grad":
        return fv.fv_distill_topk(s["logits"], s["t_ids"], s["t_logits"], tau=s["tau"], g_loss=s["g"], want_grad=True)
    r = fv.fv_distill_topk(s["logits"], s["t_ids"], s["t_logits"], tau=s["tau"])
    if s["what"] == "loss_then_grad":
        r["dlogits"] = fv.fv_distill_topk_grad(s["logits"], s["t_ids"], s["t_logits"], r["stats"], s["g"], tau=s["tau"])
    return r


# ------------------------------------------------------------------------------------------------ 64-bit definition
def exact(case, seed):
    """Row by row of the definition in float64: sums of exponentials by logsumexp, probabilities from it, gradients by
    the formulas; blocks of rows only bound the memory."""
    s = _inputs(case, seed)
    parts = []
    step = max(1, (32 << 20) // case["V"])
    for r0 in range(0, case["rows"], step):
        parts.append(_exact_rows(case, {k: v[r0:r0 + step] if torch.is_tensor(v) and k not in ("w", "b") else v for k, v in s.items()}))
    if case["op"] == "logprobs_grad":
        return torch.cat(parts)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_rows(case, s):
    tau = case["tau"]
    x = s["logits"].double() if "logits" in s else torch.einsum("rc,vc->rv", s["a"].double(), s["w"].double()) + s["b"].double()
    z = x / tau
    lse = torch.logsumexp(z, 1)
    some = lse > -math.inf
    logp = torch.where(some[:, None], z - torch.where(some, lse, torch.zeros_like(lse))[:, None], torch.full_like(z, -math.inf))
    p = logp.exp()
    m = x.max(1).values
    stats = torch.stack([m, torch.where(some, lse - m / tau, torch.full_like(lse, -math.inf))], 1)
    plogp = torch.where(p > 0, p * logp.clamp(min=-1e30), torch.zeros_like(p))
    H = -plogp.sum(1)
    r = torch.arange(x.shape[0], device=x.device)
    if case["op"] in ("logprobs", "linear"):
        ids = s["ids"].long()
        out = {"logprob": torch.where(ids >= 0, logp[r, ids.clamp(min=0)], torch.zeros_like(lse)), "stats": stats}
        if case.get("entropy", True):
            out["entropy"] = H
        if case.get("n_alt"):
            order = torch.sort(s["logits"].double(), dim=1, descending=True, stable=True).indices[:, :case["n_alt"]]
            val = torch.gather(logp, 1, order)
            out["alt_ids"] = torch.where(val > -math.inf, order, torch.full_like(order, -1)).to(torch.int32)
            out["alt_logprob"] = val
        return out
    if case["op"] == "logprobs_grad":
        ids = s["ids"].long()
        g = torch.where((ids >= 0) & some, s["g_logprob"].double(), torch.zeros_like(lse))
        dx = -g[:, None] * p
        dx[r, ids.clamp(min=0)] += g
        if s["g_entropy"] is not None:
            dx -= s["g_entropy"].double()[:, None] * (plogp + p * H[:, None])
        return dx / tau
    ids, t = s["t_ids"].long(), s["t_logits"].double() / tau
    t = torch.where(ids >= 0, t, torch.full_like(t, -math.inf))
    tl = torch.logsumexp(t, 1, keepdim=True)
    logq = t - torch.where(tl > -math.inf, tl, torch.zeros_like(tl))
    q = logq.exp()
    lp = torch.gather(logp, 1, ids.clamp(min=0))
    out = {"loss": torch.where(q > 0, q * (logq - lp), torch.zeros_like(q)).sum(1), "stats": stats}
    if case["what"] != "loss":
        dx = p * (q.sum(1, keepdim=True) > 0)
        dx.scatter_add_(1, ids.clamp(min=0), torch.where(some[:, None], -q, torch.zeros_like(q)))
        out["dlogits"] = dx * (s["g"].double() / tau)[:, None]
    return out


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(i)) for i in range(6)]:
        print(c, work(c))
