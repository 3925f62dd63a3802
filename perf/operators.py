"""The operators that teach a local head and score tokens, as timed and compared cases.

A case is a dict of plain values; prepare() makes its inputs on the GPU from a seed, run() makes one pass, work()
states the bytes and operations that the pass cannot do without and exact() computes the same outputs in float64.
With `own` set, run() calls this package's binding; otherwise it computes the operators in elementary float32
operations of torch, rounded once at the end.  Four kinds of work over rows of a vocabulary of V entries:

logprobs  logits [rows, V] -> the log probability of a given token of each row, the entropy, the log-sum-exp, and the
          top_k most likely entries with their log probabilities (by value, then by lowest index)
loss      student logits [rows, V] and a teacher's K top entries of each row (ids with logits or log probabilities)
          -> sum_k q_k (log q_k - log softmax(s / T)_k) and the log-sum-exp of s / T
grad      the same and that log-sum-exp -> the loss's gradient by the logits, weighted by one number for each row
step      loss and gradient in one call
head      the same loss for logits that are never stored, s = rho W^T: the loss alone, or with the gradients by rho
          and W

The vocabularies, ranks and rows (sequences x block positions) are those of this repository's drafting workloads and
tests; the odd ones stand for other models.  A row without teacher entries is a position that the loss leaves out.
"""
import math

import torch

own = False

V_MAIN = 151936
LOGPROBS = dict(kind="logprobs", dtype="bf16", rows=16, V=V_MAIN, pad=0, top_k=20, temperature=1.0, masked=False)
DISTILL = dict(kind="step", dtype="bf16", rows=16, V=V_MAIN, pad=0, K=64, temperature=1.0, renormalise=True, ragged=False)
HEAD = dict(kind="head", rows=1024, V=V_MAIN, r=256, K=64, temperature=1.0, renormalise=True, ragged=False, grads=True)


def listed():
    return [
        # one stream decodes one token, and its client asked for log probabilities with five alternatives
        dict(LOGPROBS, name="logprobs-1", rows=1, top_k=5),
        # one verified draft block of 16 positions, with the alternatives of a serving interface
        dict(LOGPROBS, name="logprobs-16", rows=16),
        # 64 sequences of 16 positions at once, a large serving batch
        dict(LOGPROBS, name="logprobs-1024", rows=1024),
        # a teacher's targets for distillation: 64 entries at temperature 2 of float32 rows in a padded buffer whose
        # grammar mask leaves a tenth of the vocabulary
        dict(LOGPROBS, name="logprobs-f32-300-top64", dtype="f32", rows=300, V=32003, pad=61, top_k=64, temperature=2.0,
             masked=True),
        # the smallest training step: one block of 16 positions of a small vocabulary
        dict(DISTILL, name="step-16", V=32003, K=16),
        # a validation batch in float32 against the teacher's log probabilities as they are
        dict(DISTILL, name="loss-f32-48", kind="loss", dtype="f32", rows=48, V=50003, K=20, renormalise=False),
        # the backward pass by itself, 100 teacher entries at temperature 2, some positions with fewer or none, an
        # odd vocabulary (every row starts at another alignment)
        dict(DISTILL, name="grad-777", kind="grad", rows=777, V=70001, K=100, temperature=2.0, ragged=True),
        # a training step over 128 blocks of 16 positions
        dict(DISTILL, name="step-2048", rows=2048),
        # the head's loss on a validation batch of 16 blocks
        dict(HEAD, name="head-loss-256", rows=256, K=32, grads=False),
        # a small head (rank 128) of a small vocabulary on a few blocks
        dict(HEAD, name="head-step-96", rows=96, V=32003, r=128, K=16, temperature=2.0),
        # a training step of the main head on 64 blocks
        dict(HEAD, name="head-step-1024", rows=1024),
        # the same on the positions of packed documents, some of them left out, against log probabilities
        dict(HEAD, name="head-step-6001", rows=6001, K=50, renormalise=False, ragged=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def draw(rng):
    """One more case of the same ranges."""
    pick = rng.random()
    V = rng.choice([V_MAIN, _log(rng, 5003, 152000), _log(rng, 5003, 152000)])
    if pick < 0.36:
        c = dict(LOGPROBS, dtype=rng.choice(["bf16", "bf16", "f32"]), V=V, pad=rng.choice([0, 0, 5, 64]),
                 top_k=rng.choice([0, 1, 5, 20, 20, _log(rng, 2, 128)]), temperature=rng.choice([1.0, 1.0, 0.7, 2.0]),
                 masked=rng.random() < 0.25)
        c["rows"] = min(_log(rng, 1, 1024), 150_000_000 // V)
    elif pick < 0.7:
        c = dict(DISTILL, kind=rng.choice(["loss", "grad", "step", "step"]), dtype=rng.choice(["bf16", "bf16", "f32"]), V=V,
                 pad=rng.choice([0, 0, 5, 64]), K=rng.choice([1, 16, 20, 64, _log(rng, 2, 128)]),
                 temperature=rng.choice([1.0, 1.0, 0.7, 2.0]), renormalise=rng.random() < 0.6, ragged=rng.random() < 0.4)
        c["rows"] = min(_log(rng, 4, 2048), (300_000_000 if c["dtype"] == "bf16" else 150_000_000) // V)
    else:
        c = dict(HEAD, V=V, r=rng.choice([32, 64, 128, 256, 256]), rows=_log(rng, 16, 4096), K=rng.choice([1, 16, 32, 64]),
                 temperature=rng.choice([1.0, 1.0, 2.0]), renormalise=rng.random() < 0.6, ragged=rng.random() < 0.4,
                 grads=rng.random() < 0.75)
    return c


# ----------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _logits(case, g):
    """Rows of model logits, 3 N(0, 1) with one entry raised as far as a model's confidence does, in rows of V + pad."""
    rows, V = case["rows"], case["V"]
    x = torch.empty((rows, V + case["pad"]), dtype=_dtype(case), device="cuda").normal_(0.0, 3.0, generator=g)
    top = torch.randint(0, V, (rows, 1), device="cuda", generator=g)
    lift = 4.0 + 12.0 * torch.rand((rows, 1), device="cuda", generator=g)
    x.scatter_(1, top, (x.gather(1, top).float() + lift).to(x.dtype))
    return x[:, :V], top


def _teacher(case, g):
    """A teacher's top entries: K distinct ids of each row, one from each of K ranges whose widths grow with the index
    (frequent tokens have low ids), in no order of index, with falling values.  A ragged row keeps 0 to K of them."""
    rows, V, K = case["rows"], case["V"], case["K"]
    edge = (torch.arange(K + 1, device="cuda") + (torch.arange(K + 1, device="cuda") / K) ** 3 * (V - K)).floor().long()
    u = torch.rand((rows, K), device="cuda", generator=g)
    width = edge[1:] - edge[:-1]
    ids = edge[:-1] + torch.minimum((u * width).long(), (width - 1).clamp(min=0))
    ids = ids.gather(1, torch.rand((rows, K), device="cuda", generator=g).argsort(1))
    y = 6.0 * torch.rand((rows, K), device="cuda", generator=g).sort(1, descending=True).values
    if not case["renormalise"]:   # log probabilities: the K entries hold 70% to 99% of the teacher's mass
        y = y - torch.logsumexp(y, 1, keepdim=True) + (0.7 + 0.29 * torch.rand((rows, 1), device="cuda", generator=g)).log()
    if case["ragged"]:
        kept = torch.randint(0, K + 1, (rows, 1), device="cuda", generator=g)
        ids = torch.where(torch.arange(K, device="cuda") < kept, ids, -1)
    return ids.int().contiguous(), y.float().contiguous()


def prepare(case, seed):
    g = _gen(seed)
    rows, V, T = case["rows"], case["V"], case["temperature"]
    s = dict(case=case)
    if case["kind"] == "logprobs":
        x, top = _logits(case, g)
        if case["masked"]:
            drop = torch.rand((rows, V), device="cuda", generator=g) < 0.9
            x.masked_fill_(drop.scatter_(1, top, False), -math.inf)
        s["logits"] = x
        # half of the given tokens are the likely ones
        other = torch.randint(0, V, (rows, 1), device="cuda", generator=g)
        s["tokens"] = torch.where(torch.rand((rows, 1), device="cuda", generator=g) < 0.5, top, other)[:, 0].int().contiguous()
    else:
        s["ids"], s["values"] = _teacher(case, g)
        s["weight"] = (0.5 + torch.rand(rows, device="cuda", generator=g)) / rows   # of each row in the batch's loss
        if case["kind"] == "head":
            s["rho"] = torch.empty((rows, case["r"]), dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=g)
            s["w"] = torch.empty((V, case["r"]), dtype=torch.bfloat16, device="cuda").normal_(0.0, 3.0 / math.sqrt(case["r"]), generator=g)
        else:
            x, _ = _logits(case, g)
            at = s["ids"].long().clamp(min=0)   # the student agrees with part of what the teacher expects
            agree = (torch.rand(at.shape, device="cuda", generator=g) < 0.5) & (s["ids"] >= 0)
            x.scatter_add_(1, at, torch.where(agree, 6.0, 0.0).to(x.dtype))
            s["logits"] = x
            if case["kind"] == "grad":   # the forward pass left it
                s["lse"] = torch.logsumexp(x.float() / T, 1)
    return s


# ----------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if own:
        return _run_own(s)
    if c["kind"] == "logprobs":
        return _plain_logprobs(s["logits"], s["tokens"], c["top_k"], c["temperature"])
    return _plain_distill(s)


def _run_own(s):
    from paper_2607_07409_amd import binding as B
    c = s["case"]
    if c["kind"] == "logprobs":
        stats, ids, logp = B.token_logprobs(s["logits"], s["tokens"], top_k=c["top_k"], temperature=c["temperature"])
        return dict(stats=stats, top_ids=ids, top_logprobs=logp)
    if c["kind"] == "head":
        loss, lse, d_rho, d_w = B.head_distill(s["rho"], s["w"], s["ids"], s["values"], grad_loss=s["weight"],
                                               temperature=c["temperature"], renormalise=c["renormalise"],
                                               want_grads=c["grads"])
        return dict(loss=loss, lse=lse, **(dict(d_rho=d_rho, d_w=d_w) if c["grads"] else {}))
    if c["kind"] == "grad":
        return dict(grad=B.distill_grad(s["logits"], s["lse"], s["ids"], s["values"], grad_loss=s["weight"],
                                        temperature=c["temperature"], renormalise=c["renormalise"]))
    loss, lse, grad = B.distill_loss(s["logits"], s["ids"], s["values"], grad_loss=s["weight"], temperature=c["temperature"],
                                     renormalise=c["renormalise"], want_grad=c["kind"] == "step")
    return dict(loss=loss, lse=lse, **(dict(grad=grad) if c["kind"] == "step" else {}))


def _plain_logprobs(logits, tokens, k, T):
    V = logits.shape[1]
    raw = logits.float() + 0.0   # -0 becomes 0: the two are one value
    x = raw / T
    m = x.max(1, keepdim=True).values
    e = (x - m).exp()
    z = e.sum(1, keepdim=True)
    logp = x - m - z.log()
    entropy = -torch.where(e > 0, e / z * logp, 0.0).sum(1)
    stats = torch.stack([logp.gather(1, tokens.long()[:, None])[:, 0], entropy, (m + z.log())[:, 0]], 1)
    # float32 as integers of the same order, then the lower index first: no two keys are equal
    bits = raw.contiguous().view(torch.int32)
    order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long()
    key = order * (1 << 24) + (V - 1 - torch.arange(V, device=raw.device))
    ids = key.topk(k, dim=1).indices
    return dict(stats=stats, top_ids=ids.int(), top_logprobs=logp.gather(1, ids))


def _plain_distill(s):
    c = s["case"]
    T, head = c["temperature"], c["kind"] == "head"
    if head:
        rho, w = s["rho"].float(), s["w"].float()
        x = rho @ w.T / T
    else:
        x = s["logits"].float() / T
    there = s["ids"] >= 0
    at = s["ids"].long().clamp(min=0)
    y = torch.where(there, s["values"] / T if c["renormalise"] else s["values"], -math.inf)
    if c["renormalise"]:
        top = y.max(1, keepdim=True).values.clamp(min=-1e30)
        y = y - top - (y - top).exp().sum(1, keepdim=True).clamp(min=1e-30).log()
    q = y.exp()
    out = {}
    if c["kind"] == "grad":
        lse = s["lse"][:, None]
        e, z = (x - lse).exp(), 1.0
    else:
        m = x.max(1, keepdim=True).values
        e = (x - m).exp()
        z = e.sum(1, keepdim=True)
        lse = m + z.log()
        logp = x.gather(1, at) - m - z.log()
        out = dict(loss=torch.where(q > 0, q * (y - logp), 0.0).sum(1), lse=lse[:, 0])
    if c["kind"] == "loss" or (head and not c["grads"]):
        return out
    g = s["weight"][:, None] / T
    d = g * (q.sum(1, keepdim=True) * (e / z))
    d.scatter_add_(1, at, -g * q)
    if head:
        return dict(out, d_rho=(d @ w).bfloat16(), d_w=(d.T @ rho).bfloat16())
    return dict(out, grad=d.to(s["logits"].dtype))


# ----------------------------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# ----------------------------------------------------------------------------------------------
def work(case):
    c, n = case, case["rows"] * case["V"]
    size = 4 if c.get("dtype") == "f32" else 2
    if c["kind"] == "logprobs":   # an entry: an exponential and two products summed
        return dict(bytes=n * size + c["rows"] * (16 + 8 * c["top_k"]), flops=5 * n)
    teacher = c["rows"] * (c["K"] * 8 + 12)
    if c["kind"] == "head":
        weights = c["V"] * c["r"] * 2 + c["rows"] * c["r"] * 2
        return dict(bytes=weights * (2 if c["grads"] else 1) + teacher, flops=2 * n * c["r"] * (3 if c["grads"] else 1))
    return dict(bytes=n * size * (1 if c["kind"] == "loss" else 2) + teacher, flops=(4 if c["kind"] == "loss" else 6) * n)


def exact(case, seed):
    """The definitions in float64, some rows at a time; the gradients by automatic differentiation of the loss."""
    s = prepare(case, seed)
    c = case
    rows, V, T = c["rows"], c["V"], c["temperature"]
    some = max(1, 100_000_000 // V)
    parts = [slice(a, min(rows, a + some)) for a in range(0, rows, some)]
    got = []
    if c["kind"] == "logprobs":
        for p in parts:
            x = s["logits"][p].double()
            logp = torch.log_softmax(x / T, 1)
            order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :c["top_k"]]
            entropy = torch.special.entr(logp.exp()).sum(1)
            stats = torch.stack([logp[torch.arange(len(x)), s["tokens"][p].long()], entropy, torch.logsumexp(x / T, 1)], 1)
            got.append(dict(stats=stats, top_ids=order.int(), top_logprobs=logp.gather(1, order)))
        return {k: torch.cat([d[k] for d in got]) for k in got[0]}
    step = c["kind"] in ("grad", "step") or (c["kind"] == "head" and c["grads"])
    w = s["w"].double().requires_grad_(step) if c["kind"] == "head" else None
    for p in parts:
        leaf = (s["rho"] if w is not None else s["logits"])[p].double().requires_grad_(step)
        x = (leaf @ w.T if w is not None else leaf) / T
        missing = s["ids"][p] < 0
        y = s["values"][p].double().masked_fill(missing, -math.inf)
        q = (torch.softmax(y / T, 1) if c["renormalise"] else y.exp()).masked_fill(missing, 0.0)
        lse = torch.logsumexp(x, 1)
        own_logp = x.gather(1, s["ids"][p].long().clamp(min=0)) - lse[:, None]
        if c["kind"] == "grad":   # by the log-sum-exp that the forward pass left, not by its own
            d = (x - s["lse"][p].double()[:, None]).exp() * q.sum(1, keepdim=True)
            d = d.scatter_add(1, s["ids"][p].long().clamp(min=0), -q) * (s["weight"][p].double() / T)[:, None]
            got.append(dict(grad=d.detach()))
            continue
        loss = -torch.special.entr(q).sum(1) - (q * own_logp).sum(1)
        d = dict(loss=loss.detach(), lse=lse.detach())
        if step:
            (loss * s["weight"][p].double()).sum().backward()
            d["d_rho" if w is not None else "grad"] = leaf.grad
        got.append(d)
    out = {k: torch.cat([d[k] for d in got]) for k in got[0]}
    return dict(out, d_w=w.grad) if w is not None and step else out
