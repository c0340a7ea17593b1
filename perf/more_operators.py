"""Learning against a whole pool of items, and answering from a table held in 8 bits: the calls as cases that can be timed.

`kind` says which call a case goes through:

  loss      gram_score_loss: softmax cross entropy of users against an item table from the vectors themselves, with the
            gradients of users, items and bias, the logits never kept
  quantize  gram_quantize_rows: rows of vectors to 8-bit codes with a scale for each row
  product   gram_gemm_i8: product of two such matrices, a scale for each row of either, bias, fp32 or bf16 out

loss: z[n, v] = users[n] . items[v] + bias[v]; loss[n] = -log softmax(scale z[n])[target[n]]; the gradients are those of
sum_n weight[n] loss[n].  A target of -1 means "none": loss 0, no gradient; a bias of -inf takes an item out.
quantize: inv = 127 / max |x| of the row; codes = x inv rounded to the nearest whole number (ties to even); scale = max |x| / 127.
product: C[m, n] = scale_a[m] scale_b[n] sum_k A[m, k] B[n, k] + bias[n].
"""
import functools
import math

import torch

own = False

DEV = "cuda:0"
VOCAB = 30_522                        # the encoder's vocabulary
INF = float("inf")


# --------------------------------------------------------------------------- the cases

def _loss(N, V, d, grad, bias=False, none=0.0, scale=1.0, pad=0, name=None):
    """grad: type of the vectors' gradients; none: share of the rows without a target; pad: elements between the rows' ends and starts."""
    return _named(dict(kind="loss", N=N, V=V, d=d, grad=grad, bias=bias, none=none, scale=scale, pad=pad), name)


def _quantize(N, d, dtype, pad=0, name=None):
    return _named(dict(kind="quantize", N=N, d=d, dtype=dtype, pad=pad), name)


def _product(M, N, K, out, bias=False, pad=0, name=None):
    return _named(dict(kind="product", M=M, N=N, K=K, out=out, bias=bias, pad=pad), name)


def _named(c, name):
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one student's history ends in one exercise out of the pool of 10 000: latency
        _loss(1, 10_000, 768, "bf16", name="loss_one"),
        # a short history over the smallest of the paper's pools, vectors of the small check's width, gradients for an fp32 encoder
        _loss(16, 2603, 64, "f32", name="loss_small"),
        # the news batch of 64 readers against 100 000 items with a popularity bias that takes some of them out
        _loss(64, 100_000, 768, "bf16", bias=True, name="loss_pool"),
        # a knowledge-tracing batch, 256 histories of 100 positions of which some are padding, gradients in fp32 for the encoder's backward pass
        _loss(25_600, 10_000, 768, "f32", none=0.1, name="loss_histories"),
        # masked tokens over the encoder's vocabulary
        _loss(4096, VOCAB, 768, "bf16", bias=True, name="loss_vocab"),
        # a large batch of readers against the news pool
        _loss(4096, 100_000, 768, "bf16", name="loss_large"),
        # the vectors of a batch of readers, on the way to a table's answers
        _quantize(64, 768, "bf16", name="quantize_batch"),
        # a table of 100 000 encodings, once after each training run
        _quantize(100_000, 768, "f32", name="quantize_table"),
        # one reader's logits over the table in 8 bits
        _product(1, 100_000, 768, "f32", bias=True, name="product_one"),
        # a batch of readers
        _product(64, 100_000, 768, "f32", bias=True, name="product_batch"),
        # a projection of an encoder layer (queries, keys and values) over one batch's positions
        _product(25_600, 2304, 768, "bf16", bias=True, name="product_projection"),
        # evaluation: 4096 readers over the table
        _product(4096, 100_000, 768, "bf16", name="product_eval"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["loss", "loss", "quantize", "product"])
    if kind == "loss":
        V, d, grad = _log_uniform(rng, 100, 150_000), 8 * rng.randint(2, 128), rng.choice(["bf16", "f32"])
        most = 4096 * 100_000 * 768 // (2 if grad == "f32" else 1) // (V * max(d, 128))
        N = _log_uniform(rng, 1, max(1, min(25_600, most, 4096 * 100_000 // V)))
        return _loss(N, V, d, grad, bias=rng.random() < 0.5, none=rng.choice([0.0, 0.1, 0.85]), scale=rng.choice([1.0, 0.5, 1.25]),
                     pad=rng.choice([0, 0, 8, 24]))
    if kind == "quantize":
        return _quantize(_log_uniform(rng, 1, 100_000), _log_uniform(rng, 16, 1024), rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 1, 16]))
    N, K = _log_uniform(rng, 16, 150_000), _log_uniform(rng, 16, 2048)
    M = _log_uniform(rng, 1, max(1, min(25_600, 4096 * 100_000 * 768 // (N * max(K, 768)))))
    return _product(M, N, K, rng.choice(["f32", "bf16"]) if M * N < 2048 * 100_000 else "bf16", bias=rng.random() < 0.5, pad=rng.choice([0, 0, 1, 16]))


# --------------------------------------------------------------------------- inputs

@functools.lru_cache(maxsize=None)
def _context():
    """The library's context, which a program creates once; these calls need no module in it."""
    from paper_2204_04179_b200 import binding
    cfg = binding.GramConfig()
    cfg.n_items, cfg.P_max, cfg.d = 1, 1, 8
    return binding.Gram(cfg)


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _rows(N, d, pad, dtype):
    """An [N, d] matrix whose rows lie `pad` elements further apart."""
    return torch.zeros(N, d + pad, device=DEV, dtype=dtype)[:, :d]


def _codes(N, K, g):
    """Rows in 8 bits, 16 bytes' multiple apart, and their scales, as the rows' quantisation leaves them for normal values."""
    x = torch.randn(N, K, device=DEV, generator=g)
    top = x.abs().amax(1)
    codes = torch.zeros(N, (K + 15) // 16 * 16, device=DEV, dtype=torch.int8)[:, :K]
    codes.copy_(x.mul_((127.0 / top)[:, None]).round_())
    return codes, top.mul_(0.05 / 127.0)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    st = dict(case=c)
    if c["kind"] == "loss":
        N, V, d = c["N"], c["V"], c["d"]
        # logits of deviation 3, as a model in training has them
        st["users"], st["items"] = _rows(N, d, c["pad"], torch.bfloat16), _rows(V, d, c["pad"], torch.bfloat16)
        st["users"].copy_(torch.randn(N, d, device=DEV, generator=g))
        st["items"].copy_(torch.randn(V, d, device=DEV, generator=g).mul_(3.0 / math.sqrt(d)))
        st["targets"] = torch.randint(0, V, (N,), device=DEV, generator=g, dtype=torch.int32)
        st["targets"].masked_fill_(torch.rand(N, device=DEV, generator=g) < c["none"], -1)
        st["weight"] = torch.rand(N, device=DEV, generator=g).add_(0.5).div_(N)
        st["bias"] = None
        if c["bias"]:
            st["bias"] = torch.randn(V, device=DEV, generator=g)
            st["bias"].masked_fill_(torch.rand(V, device=DEV, generator=g) < 0.01, -INF)
    elif c["kind"] == "quantize":
        st["x"] = _rows(c["N"], c["d"], c["pad"], _dtype(c["dtype"]))
        st["x"].copy_(torch.randn(c["N"], c["d"], device=DEV, generator=g))
    else:
        st["A"], st["scale_a"] = _codes(c["M"], c["K"], g)
        st["B"], st["scale_b"] = _codes(c["N"], c["K"], g)
        st["bias"] = torch.randn(c["N"], device=DEV, generator=g) if c["bias"] else None
    if own:
        gram = st["gram"] = _context()
        f = dict(device=DEV, dtype=torch.float32)
        if c["kind"] == "loss":
            grad = _dtype(c["grad"])
            st["out"] = dict(loss=torch.empty(c["N"], **f), dusers=_rows(c["N"], c["d"], c["pad"], grad), ditems=_rows(c["V"], c["d"], c["pad"], grad),
                             dbias=torch.empty(c["V"], **f) if c["bias"] else None)
            st["workspace"] = torch.empty(gram.score_loss_workspace(c["N"], c["V"], c["d"], grad)[1], device=DEV, dtype=torch.uint8)
        elif c["kind"] == "quantize":
            st["codes"] = _rows(c["N"], c["d"], -c["d"] % 16, torch.int8)
            st["scale"] = torch.empty(c["N"], **f)
        else:
            st["C"] = _rows(c["M"], c["N"], c["pad"], _dtype(c["out"]))
    return st


# --------------------------------------------------------------------------- the plain forms, in 32 bits

def _plain_loss(c, st):
    users, items, t, scale = st["users"].float(), st["items"].float(), st["targets"], c["scale"]
    z = users @ items.t()
    if st["bias"] is not None:
        z = z + st["bias"]
    y = (z - z.amax(1, keepdim=True)) * scale
    e = torch.exp(y)
    s = e.sum(1, keepdim=True)
    at = t.clamp(min=0).long()[:, None]
    live = (t >= 0)[:, None]
    logp = y.gather(1, at) - torch.log(s)
    loss = torch.where(live, -logp, torch.zeros_like(logp))[:, 0]
    w = torch.where(live & (logp > -INF), st["weight"][:, None], torch.zeros_like(logp))
    grad = e / s
    grad.scatter_add_(1, at, -torch.ones_like(logp))
    grad = grad * (w * scale)
    out = dict(loss=loss, dusers=(grad @ items).to(_dtype(c["grad"])), ditems=(grad.t() @ users).to(_dtype(c["grad"])), dbias=None)
    if st["bias"] is not None:
        out["dbias"] = grad.sum(0)
    return out


def _plain_quantize(x):
    top = x.float().abs().amax(1)
    full = torch.full_like(top, 127.0)            # quotients, not products with a reciprocal
    codes = torch.round(x.float() * (full / top)[:, None]).clamp(-127, 127).to(torch.int8)
    return dict(codes=codes, scale=top / full)


def _plain_product(c, st):
    out = (st["A"].float() @ st["B"].float().t()) * st["scale_a"][:, None] * st["scale_b"]
    if st["bias"] is not None:
        out = out + st["bias"]
    return out.to(_dtype(c["out"]))


def run(state):
    st, c = state, state["case"]
    if own:
        g = st["gram"]
        if c["kind"] == "loss":
            g.score_loss(st["users"], st["items"], st["targets"], workspace=st["workspace"], bias=st["bias"], scale=c["scale"], weight=st["weight"],
                         **st["out"])
            return st["out"]
        if c["kind"] == "quantize":
            g.quantize_rows(st["x"], st["codes"], st["scale"])
            return dict(codes=st["codes"], scale=st["scale"])
        g.gemm_i8(st["A"], st["scale_a"], st["B"], st["scale_b"], st["C"], bias=st["bias"])
        return st["C"]
    if c["kind"] == "loss":
        return _plain_loss(c, st)
    if c["kind"] == "quantize":
        return _plain_quantize(st["x"])
    return _plain_product(c, st)


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    if c["kind"] == "loss":
        N, V, d = c["N"], c["V"], c["d"]
        size = 4 if c["grad"] == "f32" else 2
        # logits, users' and items' gradient: three products; logits that are not kept are formed twice, which is not counted
        return {"bytes": (N + V) * d * (2 + size) + 12 * N + (8 * V if c["bias"] else 0), "flops": 6 * N * V * d + 10 * N * V}
    if c["kind"] == "quantize":
        return {"bytes": c["N"] * c["d"] * ((4 if c["dtype"] == "f32" else 2) + 1) + 4 * c["N"], "flops": 3 * c["N"] * c["d"]}
    M, N, K = c["M"], c["N"], c["K"]
    return {"bytes": (M + N) * (K + 4) + M * N * (4 if c["out"] == "f32" else 2) + (4 * N if c["bias"] else 0), "flops": 2 * M * N * K + 2 * M * N}


# --------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_loss(c, st):
    """The loss by logsumexp; its gradient by differentiation of that, a group of rows at a time."""
    N, V = c["N"], c["V"]
    items, bias = st["items"].double(), st["bias"]
    gone = torch.zeros(V, device=DEV, dtype=torch.bool) if bias is None else bias == -INF
    offset = torch.zeros(V, device=DEV, dtype=torch.float64) if bias is None else bias.double().masked_fill(gone, 0.0)
    loss, dusers, ditems, dbias = [], [], torch.zeros_like(items), torch.zeros_like(offset)
    per = max(1, (1 << 28) // V)
    for r in range(0, N, per):
        users, t, w = st["users"][r:r + per].double(), st["targets"][r:r + per].long(), st["weight"][r:r + per].double()
        z = (users @ items.t()).add_(offset).mul_(c["scale"]).masked_fill_(gone, -INF)
        lse = torch.logsumexp(z, 1)
        at = z.gather(1, t.clamp(min=0)[:, None])[:, 0]
        here = (lse - at).masked_fill(t < 0, 0.0)
        loss.append(here)
        w = w.masked_fill((t < 0) | (at == -INF), 0.0) * c["scale"]
        dz = z.sub_(lse[:, None]).exp_().mul_(w[:, None])
        dz[torch.arange(len(t), device=DEV), t.clamp(min=0)] -= w
        dusers.append(dz @ items)
        ditems += dz.t() @ users
        dbias += dz.sum(0)
    return dict(loss=torch.cat(loss), dusers=torch.cat(dusers), ditems=ditems, dbias=None if bias is None else dbias)


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["kind"] == "loss":
        return _exact_loss(c, st)
    if c["kind"] == "quantize":
        # the codes are whole numbers that the rounding of the 32-bit quotient decides where a value lies half way
        return dict(codes=None, scale=st["x"].double().abs().amax(1) / 127.0)
    out = (st["A"].double() @ st["B"].double().t()).mul_(st["scale_a"].double()[:, None]).mul_(st["scale_b"].double())
    return out if st["bias"] is None else out.add_(st["bias"].double())
