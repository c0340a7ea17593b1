"""Answers over a whole pool of items or a token vocabulary, and learning from them: the calls as cases that can be timed.

`kind` says which call a case goes through:

  logprobs   gram_logprobs: log probabilities of given tokens, softmax statistics, entropy, top alternatives, from logits
  backward   gram_logprobs_backward: the gradient of those log probabilities and of the entropy with respect to the logits
  distill    gram_distill: divergence from a teacher's top logits and its gradient, in one call
  score      gram_score_logprobs: the same answers as logprobs from the vectors themselves (users against an item table)

A row's logits z are scaled (x = scale z); a place at -inf is masked out: it has no probability, is never an alternative and
has no gradient.  A row with nothing left has statistics (-inf, -inf), entropy 0 and no alternatives (id -1, -inf).
A given token of -1 means "none": log probability 0.
"""
import functools
import math

import torch

own = False

DEV = "cuda:0"
VOCAB, VOCAB_LD = 30_522, 30_528      # the encoder's vocabulary, and the row stride of a product over it (a multiple of 8)
INF = float("inf")


# --------------------------------------------------------------------------- the cases

def _case(kind, N, V, dtype="f32", ld=0, C=0, k=0, scale=1.0, masked=0.0, empty=0, entropy=True, d=0, bias=False, name=None):
    """masked: share of the places at -inf; empty: every empty-th row has nothing left (0: none)."""
    c = dict(kind=kind, N=N, V=V, dtype=dtype, ld=ld or V, C=C, k=k, scale=scale, masked=masked, empty=empty, entropy=entropy, d=d, bias=bias)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one student's next exercise out of the pool of 10 000, ten suggestions: latency
        _case("logprobs", 1, 10_000, C=1, k=10, name="logprobs_one"),
        # a batch of 64 readers over 100 000 news items, the ones already read masked out, 5 candidates given
        _case("logprobs", 64, 100_000, C=5, k=10, masked=0.002, name="logprobs_pool"),
        # a teacher's lists: 4096 masked tokens over the encoder's vocabulary, 64 alternatives each
        _case("logprobs", 4096, VOCAB, "bf16", ld=VOCAB_LD, C=1, k=64, name="logprobs_vocab"),
        # cross entropy of one knowledge-tracing batch (256 histories of 100) over its 10 000 items, paddings empty
        _case("logprobs", 25_600, 10_000, C=1, empty=97, name="logprobs_histories"),
        # the gradient for one history of 100 positions
        _case("backward", 100, 10_000, C=1, entropy=False, name="backward_history"),
        # the gradient of log probability and entropy over the vocabulary
        _case("backward", 4096, VOCAB, "bf16", ld=VOCAB_LD, C=1, name="backward_vocab"),
        # the smallest of the paper's pools (2.6 thousand items, an odd number of them), one short history
        _case("distill", 16, 2603, k=10, scale=0.5, name="distill_small"),
        # 256 readers over the news pool
        _case("distill", 256, 100_000, k=64, scale=0.5, masked=0.002, name="distill_pool"),
        # a student's encoder learning the vocabulary distribution of its teacher
        _case("distill", 8192, VOCAB, "bf16", ld=VOCAB_LD, k=64, scale=0.5, empty=61, name="distill_vocab"),
        # one reader against the table of 100 000 items
        _case("score", 1, 100_000, "bf16", k=10, d=768, scale=0.05, name="score_one"),
        # the news batch against the table, with a popularity bias that takes some items out
        _case("score", 64, 100_000, "bf16", C=5, k=10, d=768, scale=0.05, bias=True, name="score_batch"),
        # evaluation: 4096 readers
        _case("score", 4096, 100_000, "bf16", C=1, k=10, d=768, scale=0.05, name="score_eval"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logprobs", "backward", "distill", "score"])
    V = _log_uniform(rng, 100, 150_000)
    scale = rng.choice([1.0, 0.5, 0.8, 1.25])
    masked = rng.choice([0.0, 0.0, 0.002, 0.1])
    empty = rng.choice([0, 0, 13, 50])
    if kind == "score":
        d = 8 * rng.randint(8, 128)
        N = _log_uniform(rng, 1, max(1, min(4096, 4096 * 100_000 * 768 // (V * d))))
        return _case(kind, N, V, "bf16", C=rng.choice([0, 1, 5]), k=rng.choice([0, 1, 10, 50]), d=d, scale=0.05 * scale,
                     bias=rng.random() < 0.5)
    dtype = rng.choice(["f32", "bf16"])
    ld = V + rng.choice([0, 0, 1, 6, (-V) % 64])
    most = {"logprobs": 25_600 * 10_000, "backward": 4096 * VOCAB, "distill": 8192 * VOCAB}[kind] // (2 if dtype == "f32" else 1)
    N = _log_uniform(rng, 1, max(1, min(25_600, most // V)))
    if kind == "logprobs":
        return _case(kind, N, V, dtype, ld, C=rng.choice([0, 1, 1, 7]), k=rng.choice([0, 1, 10, 33, 128]), scale=scale, masked=masked, empty=empty)
    if kind == "backward":
        return _case(kind, N, V, dtype, ld, C=rng.choice([1, 1, 7]), scale=scale, masked=masked, empty=empty, entropy=rng.random() < 0.5)
    return _case(kind, N, V, dtype, ld, k=rng.choice([1, 10, 64, 128]), scale=scale, masked=masked, empty=empty)


# --------------------------------------------------------------------------- inputs

@functools.lru_cache(maxsize=None)
def _context():
    """The library's context, which a program creates once; these calls need no module in it."""
    from paper_2204_04179_b200 import binding
    cfg = binding.GramConfig()
    cfg.n_items, cfg.P_max, cfg.d = 1, 1, 8
    return binding.Gram(cfg)


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _logits(c, g):
    """Logits of N rows in a buffer of row stride ld: normal with deviation 3, some places masked, some rows empty.  Returns
    (the [N, V] view, the unrounded values)."""
    N, V = c["N"], c["V"]
    z = torch.randn(N, V, device=DEV, generator=g).mul_(3.0)
    buf = torch.zeros(N, c["ld"], device=DEV, dtype=_dtype(c))
    out = buf[:, :V]
    out.copy_(z)
    if c["masked"]:
        out.masked_fill_(torch.rand(N, V, device=DEV, generator=g) < c["masked"], -INF)
    if c["empty"]:
        out[c["empty"] - 1::c["empty"]] = -INF
    return out, z


def _targets(c, g):
    """Given tokens, one in eight of them "none"."""
    t = torch.randint(0, c["V"], (c["N"], c["C"]), device=DEV, generator=g, dtype=torch.int32)
    return t.masked_fill_(torch.rand(t.shape, device=DEV, generator=g) < 0.125, -1)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    N, V = c["N"], c["V"]
    st = dict(case=c)
    if c["kind"] == "score":
        # encodings as a serving table keeps them: 8-bit codes over a common step of 1/16, held as bf16
        def code(rows):
            return torch.randn(rows, c["d"], device=DEV, generator=g).mul_(30.0).round_().clamp_(-127, 127).div_(16.0).to(torch.bfloat16)
        st["users"], st["items"] = code(N), code(V)
        # popularity in steps of 1/256; one item in a hundred is no longer offered
        st["bias"] = None
        if c["bias"]:
            st["bias"] = torch.randn(V, device=DEV, generator=g).mul_(20.0 * 256.0).round_().div_(256.0)
            st["bias"].masked_fill_(torch.rand(V, device=DEV, generator=g) < 0.01, -INF)
    else:
        st["logits"], z = _logits(c, g)
    if c["kind"] == "distill":
        # the teacher agrees with the student up to noise; its list is its k best, the last quarter of some rows unused
        a = z.mul_(0.8).add_(torch.randn(N, V, device=DEV, generator=g).mul_(2.0))
        k = min(c["k"], V)
        a, ids = a.topk(k, dim=1)
        ids = ids.to(torch.int32)
        short = (torch.rand(N, 1, device=DEV, generator=g) < 0.1) & (torch.arange(k, device=DEV) >= k - k // 4)
        st["teacher_ids"], st["teacher_logits"] = ids.masked_fill_(short, -1), a.contiguous()
        st["weight"] = torch.rand(N, device=DEV, generator=g).div_(N)
        st["weight"][N // 2:].mul_(torch.rand(N - N // 2, device=DEV, generator=g) < 0.9)
    else:
        st["targets"] = _targets(c, g) if c["C"] else None
    if c["kind"] == "backward":
        st["stats"], st["H"] = _statistics(st["logits"].float(), c["scale"])[:2]
        st["dlogp"] = torch.randn(N, c["C"], device=DEV, generator=g)
        st["dH"] = torch.rand(N, device=DEV, generator=g).mul_(0.1) if c["entropy"] else None
    if own:
        st["gram"] = _context()
        f = dict(device=DEV, dtype=torch.float32)
        if c["kind"] in ("logprobs", "score"):
            st["out"] = dict(stats=torch.empty(N, 2, **f), entropy=torch.empty(N, **f),
                             logp=torch.empty(N, c["C"], **f) if c["C"] else None,
                             top_logp=torch.empty(N, c["k"], **f) if c["k"] else None,
                             top_ids=torch.empty(N, c["k"], device=DEV, dtype=torch.int32) if c["k"] else None)
        else:
            st["dlogits"] = torch.zeros(N, c["ld"], device=DEV, dtype=_dtype(c))[:, :V]
            st["loss"] = torch.empty(N, **f)
    return st


# --------------------------------------------------------------------------- the plain forms, in 32 bits

def _statistics(z, scale):
    """(stats [N, 2], entropy [N], y = scale (z - max), e = exp(y), sum of e) of rows of logits."""
    m = z.amax(1)
    y = (z - torch.where(m == -INF, torch.zeros_like(m), m)[:, None]) * scale
    e = torch.exp(y)
    s = e.sum(1)
    log_s = torch.log(s)
    weighted = torch.where(e > 0, e * y, torch.zeros_like(e)).sum(1)
    H = torch.where(s > 0, log_s - weighted / s, torch.zeros_like(s))
    return torch.stack([m, log_s], 1), H, y, e, s


def _given(y, log_s, targets):
    """Log probabilities of the given tokens."""
    at = y.gather(1, targets.clamp(min=0).long()) - torch.where(log_s == -INF, torch.zeros_like(log_s), log_s)[:, None]
    return torch.where(targets >= 0, at, torch.zeros_like(at))


def _alternatives(z, y, log_s, k):
    """The k largest logits of each row, ties to the lowest index: (log probabilities, ids).  A logit's bits, made to order
    like a whole number, and its place form one key, so that no two keys are equal."""
    bits = (z + 0.0).view(torch.int32)
    order = bits ^ ((bits >> 31) & 0x7FFFFFFF)
    place = torch.arange(z.shape[1], device=z.device, dtype=torch.int64)
    key = (order.to(torch.int64) << 32) | (0xFFFFFFFF - place)
    top = key.topk(min(k, z.shape[1]), dim=1).values
    ids = 0xFFFFFFFF - (top & 0xFFFFFFFF)
    there = z.gather(1, ids) > -INF
    logp = torch.where(there, y.gather(1, ids) - log_s[:, None], torch.full_like(top, 1, dtype=torch.float32) * -INF)
    ids = torch.where(there, ids, -torch.ones_like(ids)).to(torch.int32)
    more = k - ids.shape[1]
    if more > 0:
        ids = torch.nn.functional.pad(ids, (0, more), value=-1)
        logp = torch.nn.functional.pad(logp, (0, more), value=-INF)
    return logp, ids


def _plain_answers(c, z, targets):
    stats, H, y, _, _ = _statistics(z, c["scale"])
    out = dict(stats=stats, entropy=H, logp=_given(y, stats[:, 1], targets) if c["C"] else None, top_logp=None, top_ids=None)
    if c["k"]:
        out["top_logp"], out["top_ids"] = _alternatives(z, y, stats[:, 1], c["k"])
    return out


def _plain_backward(c, z, stats, H, targets, dlogp, dH):
    m, log_s = stats[:, :1], stats[:, 1:]
    open_ = z > -INF
    logp = torch.where(open_, (z - m) * c["scale"] - log_s, torch.full_like(z, -INF))
    p = torch.exp(logp)
    t = targets.clamp(min=0).long()
    g = torch.where((targets >= 0) & open_.gather(1, t), dlogp, torch.zeros_like(dlogp))
    dz = -p * g.sum(1, keepdim=True)
    if dH is not None:
        dz -= torch.where(p > 0, p * (logp + H[:, None]), torch.zeros_like(p)) * dH[:, None]
    dz.scatter_add_(1, t, g)
    return dz * c["scale"]


def _plain_distill(c, z, ids, a, weight):
    stats, _, y, e, s = _statistics(z, c["scale"])
    t = ids.clamp(min=0).long()
    use = (ids >= 0) & (z.gather(1, t) > -INF)
    a = torch.where(use, a * c["scale"], torch.full_like(a, -INF))
    a_max = a.amax(1, keepdim=True)
    some = a_max > -INF
    ya = a - torch.where(some, a_max, torch.zeros_like(a_max))
    ea = torch.exp(ya)
    total = ea.sum(1, keepdim=True)
    zero = torch.zeros_like(ea)
    q = torch.where(some, ea / total, zero)
    log_q = ya - torch.log(total)
    logp = y.gather(1, t) - stats[:, 1:]
    loss = torch.where(q > 0, q * (log_q - logp), zero).sum(1)
    dz = torch.where(some, e / s[:, None], torch.zeros_like(e))
    dz.scatter_add_(1, t, -q)
    return dict(loss=loss, dlogits=dz * (weight * c["scale"])[:, None])


def run(state):
    st, c = state, state["case"]
    kind = c["kind"]
    if own:
        g = st["gram"]
        if kind == "logprobs":
            g.logprobs(st["logits"], scale=c["scale"], targets=st["targets"], **st["out"])
            return st["out"]
        if kind == "score":
            g.score_logprobs(st["users"], st["items"], bias=st["bias"], scale=c["scale"], targets=st["targets"], **st["out"])
            return st["out"]
        if kind == "backward":
            g.logprobs_backward(st["logits"], st["stats"], st["dlogits"], scale=c["scale"], targets=st["targets"],
                                dlogp=st["dlogp"], entropy=st["H"] if st["dH"] is not None else None, dentropy=st["dH"])
            return dict(dlogits=st["dlogits"])
        g.distill(st["logits"], st["teacher_ids"], st["teacher_logits"], st["loss"], scale=c["scale"], weight=st["weight"],
                  dlogits=st["dlogits"])
        return dict(loss=st["loss"], dlogits=st["dlogits"])
    if kind == "logprobs":
        return _plain_answers(c, st["logits"].float(), st["targets"])
    if kind == "score":
        z = st["users"].float() @ st["items"].float().t()
        if st["bias"] is not None:
            z = z + st["bias"]
        return _plain_answers(c, z, st["targets"])
    if kind == "backward":
        dz = _plain_backward(c, st["logits"].float(), st["stats"], st["H"], st["targets"], st["dlogp"], st["dH"])
        return dict(dlogits=dz.to(st["logits"].dtype))
    out = _plain_distill(c, st["logits"].float(), st["teacher_ids"], st["teacher_logits"], st["weight"])
    return dict(loss=out["loss"], dlogits=out["dlogits"].to(st["logits"].dtype))


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    N, V, C, k = c["N"], c["V"], c["C"], c["k"]
    size = 4 if c["dtype"] == "f32" else 2
    answers = N * (12 + 8 * C + 8 * k)                # statistics and entropy; given tokens in and out; alternatives
    if c["kind"] == "logprobs":
        return {"bytes": N * V * size + answers, "flops": 6 * N * V}
    if c["kind"] == "backward":
        return {"bytes": 2 * N * V * size + N * (8 * C + 16), "flops": 8 * N * V}
    if c["kind"] == "distill":
        return {"bytes": 2 * N * V * size + N * (8 * k + 8), "flops": 8 * N * V}
    return {"bytes": (N + V) * c["d"] * 2 + (4 * V if c["bias"] else 0) + answers, "flops": 2 * N * V * c["d"] + 6 * N * V}


# --------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_answers(c, z, targets):
    """z: float64 rows."""
    x = c["scale"] * z
    lse = torch.logsumexp(x, 1)
    dead = lse == -INF
    logp = x - lse.masked_fill(dead, 0.0)[:, None]
    p = logp.exp()
    m = z.max(1).values
    out = dict(stats=torch.stack([m, (lse - c["scale"] * m).masked_fill(dead, -INF)], 1), entropy=torch.special.entr(p).sum(1),
               logp=None, top_logp=None, top_ids=None)
    if c["C"]:
        rows = torch.arange(z.shape[0], device=z.device)[:, None]
        out["logp"] = logp[rows, targets.long()].masked_fill(targets < 0, 0.0)
    if c["k"]:
        n = min(c["k"], z.shape[1])
        val, at = torch.sort(z, dim=1, descending=True, stable=True)
        val, at = val[:, :n], at[:, :n]
        ids = torch.full((z.shape[0], c["k"]), -1, device=z.device, dtype=torch.int32)
        ids[:, :n] = at.masked_fill(val == -INF, -1).to(torch.int32)
        top = torch.full((z.shape[0], c["k"]), -INF, device=z.device, dtype=torch.float64)
        top[:, :n] = logp.gather(1, at)
        out["top_logp"], out["top_ids"] = top, ids
    return out


def _exact_gradient(c, z, targets, dlogp, dH):
    """By differentiation of the definition, masked places held constant."""
    at = z.gather(1, targets.clamp(min=0).long())
    live = (targets >= 0) & (at > -INF)
    leaf = z.masked_fill(z == -INF, 0.0).requires_grad_()
    x = (c["scale"] * leaf).masked_fill(z == -INF, -INF)
    x = torch.where((z == -INF).all(1, keepdim=True), torch.zeros_like(x), x)
    logp = x - torch.logsumexp(x, 1, keepdim=True)
    total = (logp.gather(1, targets.clamp(min=0).long()).masked_fill(~live, 0.0) * dlogp.double()).sum()
    if dH is not None:
        safe = logp.masked_fill(z == -INF, 0.0)
        total = total - ((safe.exp() * safe).masked_fill(z == -INF, 0.0).sum(1) * dH.double()).sum()
    return torch.autograd.grad(total, leaf)[0].masked_fill(z == -INF, 0.0)


def _exact_distill(c, z, ids, a, weight):
    at = z.gather(1, ids.clamp(min=0).long())
    a = (c["scale"] * a.double()).masked_fill((ids < 0) | (at == -INF), -INF)
    some = (a > -INF).any(1, keepdim=True)
    q = torch.softmax(a.masked_fill(~some, 0.0), 1) * some
    x = (c["scale"] * z).masked_fill(~some, 0.0)
    logp = x - torch.logsumexp(x, 1, keepdim=True)
    got = logp.gather(1, ids.clamp(min=0).long())
    loss = (torch.xlogy(q, q) - q * got.masked_fill(q == 0, 0.0)).sum(1)
    dz = logp.exp() * some
    dz.scatter_add_(1, ids.clamp(min=0).long(), -q)
    return dict(loss=loss, dlogits=dz * (c["scale"] * weight.double())[:, None])


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    per = max(1, (1 << 26) // c["V"])                 # rows at a time, so that the 64-bit copies stay small
    parts = []
    for r in range(0, c["N"], per):
        cut = {k: v[r:r + per] if torch.is_tensor(v) and k not in ("items", "bias") else v for k, v in st.items()}
        if c["kind"] == "score":
            z = cut["users"].double() @ cut["items"].double().t()
            if cut["bias"] is not None:
                z += cut["bias"].double()
            parts.append(_exact_answers(c, z, cut["targets"]))
            continue
        z = cut["logits"].double()
        if c["kind"] == "logprobs":
            parts.append(_exact_answers(c, z, cut["targets"]))
        elif c["kind"] == "backward":
            parts.append(dict(dlogits=_exact_gradient(c, z, cut["targets"], cut["dlogp"], cut["dH"])))
        else:
            parts.append(_exact_distill(c, z, cut["teacher_ids"], cut["teacher_logits"], cut["weight"]))
    return {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}
