"""Gradients of dls_head_distill for a student that agrees with its teacher, against float64: confident rows (the likeliest
token holds 0.9 to 0.999 of the mass), the teacher's entries the student's own likeliest tokens with almost its
probabilities, so that g / T (M p - q) is a small difference of large numbers.

Tolerances (u = 2^-24).  A logit sums r exact products in float32, within u r |rho|.|W|, and is scaled and referred with a
rounding each: within e = u (V / 32 + 40) + 4 u |x|max + u r |rho|.|W| / T of the float64 one relative to the log-sum-exp (as
test_head_distill.py), and q is within 8 u (1 + span of the values): E = 2 e + 8 u (1 + span) bounds what either is off by,
relative to itself.  Only probabilities of tokens that the teacher does not name are rounded to bf16, and the result once,
each within 2^-8 (8 significant bits).  Entry by entry a gradient is within
  2^-8 sum_{v not named} |M p_v W_v| + 2^-8 |result| + E sum_v (M p_v + q_v) |W_v|
(weighted by |g / T|; d_W the same over the rows).
"""
import math

import pytest
import torch

from paper_2607_07409_amd import binding as B

U = 2.0 ** -24
BF16 = torch.bfloat16


def _agreeing(rows, V, r, K, top_p, seed, T=1.0, tokens=None, noise=0.05, renorm=True, twice=False):
    """rho, W, ids, values, weight: one token of each row lifted to the share top_p at temperature T."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, device="cuda", generator=g)   # noqa: E731
    w = (normal(V, r) * (2.0 * T / math.sqrt(r))).to(BF16)
    rho = normal(rows, r)
    tok = torch.randint(0, tokens or V, (rows,), device="cuda", generator=g)
    for _ in range(3):   # (the shift changes the other logits a little)
        x = rho.double() @ w.double().T / T
        others = torch.logsumexp(x.scatter(1, tok[:, None], -math.inf), 1)
        lift = others + math.log(top_p / (1 - top_p)) - x.gather(1, tok[:, None])[:, 0]
        wt = w[tok].double()
        rho = (rho.double() + wt * (lift * T / wt.pow(2).sum(1))[:, None]).float()
    rho = rho.to(BF16)
    x = rho.double() @ w.double().T / T
    ids = x.topk(K // 2 if twice else K, 1).indices
    ids = ids[:, torch.randperm(ids.shape[1], device="cuda", generator=g)]
    logp = (x - torch.logsumexp(x, 1, keepdim=True)).gather(1, ids) + noise * normal(*ids.shape).double()
    y = (logp * (T if renorm else 1.0)).float()
    if not renorm:   # (no more mass than there is)
        y -= torch.logsumexp(y, 1, keepdim=True).clamp(min=0)
    if twice:        # each entry as two with half its weight
        ids, y = ids.repeat(1, 2), y.repeat(1, 2) - (0.0 if renorm else math.log(2.0))
    return rho, w, ids.int().contiguous(), y.contiguous(), (0.5 + torch.rand(rows, device="cuda", generator=g)) * torch.sign(normal(rows))


def _check(rho, w, ids, y, weight, T, renorm, d_rho, d_w):
    V, r = w.shape
    at = ids.long()
    a, b = rho.double(), w.double()
    x = a @ b.T / T
    lse = torch.logsumexp(x, 1, keepdim=True)
    yd = y.double()
    q = torch.softmax(yd / T, 1) if renorm else yd.exp()
    g = (weight.double() / T)[:, None]
    p = (x - lse).exp() * q.sum(1, keepdim=True)
    full = torch.zeros_like(p).scatter_add_(1, at, q)
    d = g * (p - full)
    span = float((yd.max(1).values - yd.min(1).values).max()) / T
    size = float(a.norm(dim=1).max() * b.norm(dim=1).max()) / T
    e = U * (V / 32 + 40) + 4 * U * float(x.abs().max()) + U * r * size
    both = 2 * e + 8 * U * (1 + span)
    dense = p.scatter(1, at, 0.0) * g.abs()
    share = both * (p + full) * g.abs()
    report = []
    for name, got, want, tol in (("d_rho", d_rho, d @ b, (2.0 ** -8 * dense + share) @ b.abs()),
                                 ("d_w", d_w, d.T @ a, (2.0 ** -8 * dense + share).T @ a.abs())):
        tol = tol + 2.0 ** -8 * want.abs() + 1e-30
        off = (got.double() - want).abs()
        report.append((name, float(off.norm() / want.norm()), float(tol.norm() / want.norm()), int((off > tol).sum())))
    print(report)
    assert all(bad == 0 for *_, bad in report), report
    return report


@pytest.mark.gpu
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("top_p", [0.9, 0.99, 0.999])
@pytest.mark.parametrize("rows,V,r,K", [(256, 8000, 128, 64), (70, 3001, 64, 20), (300, 10007, 256, 32), (40, 1999, 136, 256)])
def test_agreeing_student(rows, V, r, K, top_p, renorm):
    c = _agreeing(rows, V, r, K, top_p, rows + K, renorm=renorm)
    _, _, d_rho, d_w = B.head_distill(*c[:4], grad_loss=c[4], renormalise=renorm, want_grads=True)
    _check(*c, 1.0, renorm, d_rho, d_w)


@pytest.mark.gpu
@pytest.mark.parametrize("r", [64, 128, 256])
@pytest.mark.parametrize("rows,V", [(600, 1500), (2100, 600)])
def test_few_tokens_of_many_rows(rows, V, r):
    """Tokens that many rows share: long lists of few, also where the rows of a tile of W are shared by workgroups."""
    c = _agreeing(rows, V, r, 24, 0.99, 7, tokens=9)
    _, _, d_rho, d_w = B.head_distill(*c[:4], grad_loss=c[4], want_grads=True)
    _check(*c, 1.0, True, d_rho, d_w)


@pytest.mark.gpu
@pytest.mark.parametrize("r", [64, 128, 256])
def test_repeated_ids(r):
    """An id that the teacher names twice takes its probability's exact part once."""
    c = _agreeing(130, 3001, r, 16, 0.99, 11, renorm=False, twice=True)
    _, _, d_rho, d_w = B.head_distill(*c[:4], grad_loss=c[4], renormalise=False, want_grads=True)
    _check(*c, 1.0, False, d_rho, d_w)


@pytest.mark.gpu
@pytest.mark.parametrize("r", [64, 128, 256])
def test_the_likeliest_token_at_the_end(r):
    """Logits that rise by hundreds towards the vocabulary's end, where the teacher's tokens are."""
    rows, V, K = 70, 4099, 16
    rho, w, _, _, weight = _agreeing(rows, V, r, K, 0.9, 13)
    direction = torch.sign(rho[0].float())
    rho = (rho.float().abs() * direction).to(BF16)
    w = (w.float() + torch.linspace(-1.0, 1.0, V, device="cuda")[:, None] * direction * (300.0 / r)).to(BF16)
    for w in (w, w.flip(0).contiguous()):
        x = rho.double() @ w.double().T
        best = x.topk(K, 1)
        y = (best.values - torch.logsumexp(x, 1, keepdim=True)).float() + 0.05 * torch.randn((rows, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
        ids = best.indices.int().contiguous()
        _, _, d_rho, d_w = B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True)
        _check(rho, w, ids, y, weight, 1.0, True, d_rho, d_w)
