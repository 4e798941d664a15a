"""The operators at the vocabulary's two ends of a policy-gradient pass: what they compute, in plain form
and through the library, and the sizes they are measured at.

  logprobs       log-probs of given tokens from logits, with entropy and the most likely alternatives
  logprobs_grad  the logits' gradient from those of the log-probs and entropies
  embed          embedding lookup with scaling
  embed_grad     the embedding matrix's gradient
  head           log-probs and entropies straight from hidden states and the lm_head matrix
  head_grad      the gradients of both

Vocabularies and hidden sizes are those of the benchmark's configurations and of the small test shapes, rows
those of decode steps (1 to a few hundred) and of packed sequences (thousands).  A quarter of the rows of a
gradient call are prompt tokens, which have no gradient.  Logits spread as a trained model's: the given token
is usually among the likely ones.
"""
import math

import torch

import paper_2506_06122_amd as R

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
VOCABS = [1024, 4096, 32001, 50257, 151936, 152064]


# ---------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one sample of a decode step: log-prob, entropy and 20 alternatives of a single row
        dict(name="logprobs_one_token", kind="logprobs", rows=1, vocab=151936, dtype="fp32", top=20, temperature=1.0,
             pad=0, banned=True),
        # packed sequences of a training batch, alternatives kept for distillation
        dict(name="logprobs_batch", kind="logprobs", rows=2048, vocab=152064, dtype="bf16", top=8, temperature=0.7,
             pad=0, banned=False),
        # a small model's micro-batch, rows inside wider ones
        dict(name="logprobs_grad_small", kind="logprobs_grad", rows=61, vocab=32001, dtype="fp16", entropy=False,
             temperature=1.0, pad=63),
        # the logits' gradient of a training batch, with an entropy bonus
        dict(name="logprobs_grad_batch", kind="logprobs_grad", rows=6144, vocab=152064, dtype="bf16", entropy=True,
             temperature=1.0, pad=0),
        # the live rows of a decode step
        dict(name="embed_step", kind="embed", tokens=187, vocab=151936, hidden=1536, dtype="bf16", scale=1.0),
        # packed sequences of a training batch
        dict(name="embed_batch", kind="embed", tokens=16384, vocab=152064, hidden=3584, dtype="bf16", scale=59.875),
        # a tied matrix: the lookup's gradient on top of the head's, in single precision
        dict(name="embed_grad_tied", kind="embed_grad", tokens=1021, vocab=4096, hidden=1536, dtype="bf16", out="fp32",
             base=True, scale=1.0),
        # the whole gradient of a large vocabulary's embedding
        dict(name="embed_grad_batch", kind="embed_grad", tokens=16384, vocab=152064, hidden=3584, dtype="bf16",
             out="bf16", base=False, scale=59.875),
        # a few rows: a walk over the matrix
        dict(name="head_few", kind="head", rows=7, vocab=151936, hidden=1536, temperature=1.0),
        # a training micro-batch of the larger dense model
        dict(name="head_batch", kind="head", rows=4096, vocab=152064, hidden=3584, temperature=1.0),
        # a short packed batch of the smaller dense model
        dict(name="head_grad_short", kind="head_grad", rows=613, vocab=151936, hidden=1536, temperature=0.7,
             entropy=True),
        # a training micro-batch of the larger dense model
        dict(name="head_grad_batch", kind="head_grad", rows=4096, vocab=152064, hidden=3584, temperature=1.0,
             entropy=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logprobs", "logprobs_grad", "embed", "embed_grad", "head", "head_grad"])
    vocab = rng.choice(VOCABS)
    temperature = rng.choice([0.6, 0.7, 1.0, 1.0, 1.3])
    if kind == "logprobs":
        return dict(kind=kind, rows=_log(rng, 1, 2048), vocab=vocab, dtype=rng.choice(list(TYPES)),
                    top=rng.choice([0, 1, 5, 20, 64]), temperature=temperature, pad=rng.choice([0, 0, 1, 64]),
                    banned=rng.random() < 0.5)
    if kind == "logprobs_grad":
        return dict(kind=kind, rows=_log(rng, 1, 4096), vocab=vocab, dtype=rng.choice(list(TYPES)),
                    entropy=rng.random() < 0.5, temperature=temperature, pad=rng.choice([0, 0, 1, 64]))
    hidden = rng.choice([128, 512, 1536, 2048, 3584])
    if kind == "embed":
        return dict(kind=kind, tokens=_log(rng, 1, 16384), vocab=vocab, hidden=hidden, dtype=rng.choice(list(TYPES)),
                    scale=rng.choice([1.0, round(math.sqrt(hidden), 3)]))
    if kind == "embed_grad":
        dtype = rng.choice(list(TYPES))
        return dict(kind=kind, tokens=_log(rng, 1, 16384), vocab=vocab, hidden=hidden, dtype=dtype,
                    out=rng.choice(["fp32", dtype]), base=rng.random() < 0.3,
                    scale=rng.choice([1.0, round(math.sqrt(hidden), 3)]))
    c = dict(kind=kind, rows=_log(rng, 1, 4096), vocab=vocab, hidden=hidden, temperature=temperature)
    return c if kind == "head" else dict(c, entropy=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------- inputs
def _masked(n, gen):
    """A quarter of the rows: the prompt tokens."""
    m = torch.zeros(n, dtype=torch.bool, device="cuda")
    m[torch.randperm(n, device="cuda", generator=gen)[:n // 4]] = True
    return m


def _row_grads(c, n, gen):
    """d loss / d logp of a token-mean loss over clipped advantages, and of an entropy bonus."""
    masked = _masked(n, gen)
    g = torch.randn(n, device="cuda", generator=gen).clamp_(-10, 10) / -n
    h = torch.full((n,), -0.01 / n, device="cuda") if c["entropy"] else None
    return g.masked_fill_(masked, 0.0), None if h is None else h.masked_fill_(masked, 0.0)


def _forward(x, inv_t):
    """(d, ln S, p, entropy, row stats) of float logits."""
    m = x.max(1, keepdim=True).values
    d = (x - m) * inv_t
    e = d.exp()
    total = e.sum(1, keepdim=True)
    log_s = total.log()
    p = e / total
    entropy = log_s[:, 0] - torch.where(p > 0, p * d, torch.zeros((), device=x.device)).sum(1)
    return d, log_s, p, entropy, torch.cat([m, log_s], 1)


def _head_inputs(c, gen):
    rows, vocab, hidden = c["rows"], c["vocab"], c["hidden"]
    w = torch.empty(vocab, hidden, device="cuda", dtype=torch.bfloat16).normal_(0.0, 2.5 / math.sqrt(hidden), generator=gen)
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
    h = torch.randn(rows, hidden, device="cuda", generator=gen)
    h += w[t].float() * torch.rand(rows, 1, device="cuda", generator=gen) * 2.0  # up to +12.5 on the given token
    return h.to(torch.bfloat16), w, t.int()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": c, "inv_t": 1.0 / c.get("temperature", 1.0)}
    kind = c["kind"]
    if kind in ("logprobs", "logprobs_grad"):
        rows, vocab = c["rows"], c["vocab"]
        x = torch.empty(rows, vocab + c["pad"], device="cuda", dtype=TYPES[c["dtype"]])[:, :vocab]
        x.normal_(0.0, 2.5, generator=gen)
        t = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
        lift = torch.rand(rows, 1, device="cuda", generator=gen) * 14.0
        x.scatter_(1, t[:, None], (x.gather(1, t[:, None]).float() + lift).to(x.dtype))
        if c.get("banned"):  # ids that may not be drawn, the given token never among them
            off = torch.randint(0, vocab, (vocab // 50,), device="cuda", generator=gen)
            keep = x.gather(1, t[:, None])
            x[:, off] = float("-inf")
            x.scatter_(1, t[:, None], keep)
        s.update(x=x, targets=t.int())
        if kind == "logprobs_grad":
            _, _, _, entropy, stats = _forward(x.float(), s["inv_t"])
            g, h = _row_grads(c, rows, gen)
            s.update(stats=stats, entropy=entropy, g=g, h=h)
        return s
    if kind in ("embed", "embed_grad"):
        n, vocab, hidden = c["tokens"], c["vocab"], c["hidden"]
        # a few ids are most of the text; some rows are padding
        ids = (torch.rand(n, device="cuda", generator=gen) ** 4 * vocab).int().clamp_(max=vocab - 1)
        ids[torch.rand(n, device="cuda", generator=gen) < 0.05] = 13 % vocab
        ids[torch.rand(n, device="cuda", generator=gen) < 0.02] = -1
        s["ids"] = ids
        if kind == "embed":
            s["table"] = torch.empty(vocab, hidden, device="cuda", dtype=TYPES[c["dtype"]]).normal_(0.0, 0.02, generator=gen)
            return s
        s["dy"] = torch.empty(n, hidden, device="cuda", dtype=TYPES[c["dtype"]]).normal_(0.0, 0.01, generator=gen)
        s["base"] = (torch.empty(vocab, hidden, device="cuda", dtype=TYPES[c["out"]]).normal_(0.0, 0.01, generator=gen)
                     if c["base"] else None)
        return s
    h, w, t = _head_inputs(c, gen)
    s.update(hidden=h, w=w, targets=t)
    if kind == "head_grad":
        _, _, _, entropy, stats = _forward(h.float() @ w.float().T, s["inv_t"])
        g, e = _row_grads(c, c["rows"], gen)
        s.update(stats=stats, entropy=entropy, g=g, h=e)
    return s


# ---------------------------------------------------------------------------------------- one pass
def _plain_logprobs(x, targets, inv_t, top):
    d, log_s, _, entropy, stats = _forward(x, inv_t)
    logp = d.gather(1, targets.long()[:, None])[:, 0] - log_s[:, 0]
    out = [logp, entropy, stats]
    if top:
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
        out += [ids.int(), d.gather(1, ids) - log_s]
    return out


def _plain_dx(x, s):
    """The logits' gradient in 32 bits."""
    inv_t = s["inv_t"]
    lp = (x - s["stats"][:, :1]) * inv_t - s["stats"][:, 1:]
    p = lp.exp()
    dx = p * -s["g"][:, None]
    if s["h"] is not None:
        dx -= torch.where(p > 0, p * (lp + s["entropy"][:, None]), torch.zeros((), device=x.device)) * s["h"][:, None]
    t = s["targets"].long()[:, None]
    dx.scatter_add_(1, t, s["g"][:, None])
    return dx * inv_t


def run(state):
    s, c = state, state["case"]
    kind, temperature = c["kind"], c.get("temperature", 1.0)
    if kind == "logprobs":
        if own:
            out = R.rollout_token_logprobs(s["x"], s["targets"], temperature=temperature, top=c["top"])
            return list(out[:5] if c["top"] else out[:3])
        return _plain_logprobs(s["x"].float(), s["targets"], s["inv_t"], c["top"])
    if kind == "logprobs_grad":
        if own:
            return R.rollout_token_logprobs_grad(s["x"], s["targets"], s["stats"], s["entropy"], s["g"], s["h"],
                                                 temperature=temperature)
        return _plain_dx(s["x"].float(), s).to(s["x"].dtype)
    if kind == "embed":
        if own:
            return R.rollout_embed(s["table"], s["ids"], scale=c["scale"])
        rows = s["table"][s["ids"].long().clamp(min=0)].float() * c["scale"]
        return rows.masked_fill_(s["ids"][:, None] < 0, 0.0).to(s["table"].dtype)
    if kind == "embed_grad":
        out_type = TYPES[c["out"]]
        if own:
            return R.rollout_embed_grad(s["dy"], s["ids"], c["vocab"], scale=c["scale"], base=s["base"], dtype=out_type)
        acc = torch.zeros(c["vocab"], c["hidden"], device="cuda")
        dy = s["dy"].float().masked_fill_(s["ids"][:, None] < 0, 0.0)
        acc.index_add_(0, s["ids"].long().clamp(min=0), dy)
        acc *= c["scale"]
        if s["base"] is not None:
            acc += s["base"].float()
        return acc.to(out_type)
    if kind == "head":
        if own:
            return list(R.rollout_head_logprobs(s["hidden"], s["w"], s["targets"], temperature=temperature))
        return _plain_logprobs(s["hidden"].float() @ s["w"].float().T, s["targets"], s["inv_t"], 0)
    if own:
        return list(R.rollout_head_logprobs_grad(s["hidden"], s["w"], s["targets"], s["stats"], s["entropy"], s["g"],
                                                 s["h"], temperature=temperature))
    h, w = s["hidden"].float(), s["w"].float()
    dx = _plain_dx(h @ w.T, s)
    return [(dx @ w).to(torch.bfloat16), (dx.T @ h).to(torch.bfloat16)]


# ---------------------------------------------------------------------------------------- in 64 bits
def _exact_rows(x, c):
    """(log-softmax with temperature, entropy) of logits in double precision."""
    z = x / c["temperature"]
    lp = z - torch.logsumexp(z, 1, keepdim=True)
    return lp, -(lp.exp() * lp.clamp(min=-1e30)).sum(1)


def _exact_dx(x, s, c):
    """d/dx of sum_r g_r logp_r + h_r entropy_r, from the derivative of log-softmax."""
    lp, entropy = _exact_rows(x, c)
    p = lp.exp()
    up = -s["h"].double()[:, None] * p * (lp.clamp(min=-1e30) + entropy[:, None]) if s["h"] is not None else torch.zeros_like(p)
    up -= s["g"].double()[:, None] * p
    rows = torch.arange(len(p), device="cuda")
    up[rows, s["targets"].long()] += s["g"].double()
    return up / c["temperature"]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    kind = c["kind"]
    if kind == "logprobs" or kind == "head":
        x = s["x"].double() if kind == "logprobs" else s["hidden"].double() @ s["w"].double().T
        lp, entropy = _exact_rows(x, c)
        rows = torch.arange(len(x), device="cuda")
        top = x.amax(1)
        stats = torch.stack([top, torch.logsumexp((x - top[:, None]) / c["temperature"], 1)], 1)
        out = [lp[rows, s["targets"].long()], entropy, stats]
        if c.get("top"):
            order = torch.topk(x, c["top"], dim=1).values  # the values are the same however ties are ordered
            out += [None, order / c["temperature"] - torch.logsumexp(x / c["temperature"], 1, keepdim=True)]
        return out
    if kind == "logprobs_grad":
        return _exact_dx(s["x"].double(), s, c)
    if kind == "embed":
        out = torch.zeros(c["tokens"], c["hidden"], dtype=torch.float64, device="cuda")
        here = s["ids"] >= 0
        out[here] = s["table"].double()[s["ids"][here].long()] * c["scale"]
        return out
    if kind == "embed_grad":
        here = s["ids"] >= 0
        out = s["base"].double() if s["base"] is not None else torch.zeros(c["vocab"], c["hidden"], dtype=torch.float64,
                                                                           device="cuda")
        return out.index_put_((s["ids"][here].long(),), s["dy"][here].double() * c["scale"], accumulate=True)
    h, w = s["hidden"].double(), s["w"].double()
    dx = _exact_dx(h @ w.T, s, c)
    return [dx @ w, dx.T @ h]


# ---------------------------------------------------------------------------------------- what it takes
def work(case):
    c = case
    kind = c["kind"]
    size = {"fp32": 4, "bf16": 2, "fp16": 2}
    if kind in ("logprobs", "logprobs_grad"):
        rows, values = c["rows"], float(c["rows"]) * c["vocab"]
        if kind == "logprobs":
            return {"bytes": values * size[c["dtype"]] + rows * (20.0 + 8.0 * c["top"]), "flops": 8.0 * values}
        read = values * (rows - rows // 4) / rows
        return {"bytes": (read + values) * size[c["dtype"]] + 24.0 * rows, "flops": 8.0 * read}
    if kind in ("embed", "embed_grad"):
        values = float(c["tokens"]) * c["hidden"]
        if kind == "embed":
            return {"bytes": 2.0 * values * size[c["dtype"]] + 4.0 * c["tokens"], "flops": values}
        whole = float(c["vocab"]) * c["hidden"] * size[c["out"]]
        return {"bytes": values * size[c["dtype"]] + whole * (2 if c["base"] else 1) + 4.0 * c["tokens"], "flops": values}
    rows, hv = c["rows"], float(c["hidden"]) * c["vocab"]
    moved = 2.0 * (hv + rows * c["hidden"]) + 24.0 * rows
    if kind == "head":
        return {"bytes": moved, "flops": 2.0 * rows * hv}
    return {"bytes": 2.0 * moved, "flops": 6.0 * (rows - rows // 4) * hv}
