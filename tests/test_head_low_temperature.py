"""dls_head_distill at low temperatures and with logits far from 0: s / T of 10^4 to 10^6, where a float32 number holds few
digits after the point, though the differences that the probabilities are made of are exact.

States and weights are chosen so that every logit is exact in float32 (one column gives an offset, the others multiples of a
power of two), so a probability is as good as its distance to the row's largest logit, span = max x - min x at most: within
e = u (V / 32 + 40) + 4 u span of itself (u = 2^-24; additions of one lane, one rounding of the distance, the exponential).  The
gradients then follow test_head_agreement.py with this e.
"""
import pytest
import torch

from paper_2607_07409_amd import binding as B

U = 2.0 ** -24
BF16 = torch.bfloat16


def _make(rows, V, r, K, T, offset, seed):
    g = torch.Generator().manual_seed(seed)
    third = lambda *shape: torch.randint(-1, 2, shape, generator=g).float()   # noqa: E731
    rho, w = third(rows, r) * (2.0 ** 6 * T), third(V, r) * 2.0 ** -7
    rho[:, 0], w[:, 0] = 8.0, offset / 8.0
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(rows)]).int()
    y = torch.randn((rows, K), generator=g) * (2 * T)
    weight = torch.randn(rows, generator=g)
    return rho.to(BF16).cuda(), w.to(BF16).cuda(), ids.cuda(), y.cuda(), weight.cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2.0 ** -13, 2.0 ** -10, 2.0 ** -7])
@pytest.mark.parametrize("offset", [0.0, 16.0, -64.0, 256.0])
@pytest.mark.parametrize("rows,V,r", [(60, 2001, 64), (300, 5003, 128), (90, 1999, 256)])
def test_far_logits_at_low_temperature(rows, V, r, offset, T):
    K = 16
    rho, w, ids, y, weight = _make(rows, V, r, K, T, offset, rows)
    _, _, d_rho, d_w = B.head_distill(rho, w, ids, y, grad_loss=weight, temperature=T, want_grads=True)
    a, b, at = rho.double(), w.double(), ids.long()
    s = a @ b.T
    assert torch.equal(s, s.float().double())
    x = s / T
    q = torch.softmax(y.double() / T, 1)
    g = (weight.double() / T)[:, None]
    p = torch.softmax(x, 1)
    full = torch.zeros_like(p).scatter_add_(1, at, q)
    d = g * (p - full)
    span = float((x.max(1).values - x.min(1).values).max())
    e = U * (V / 32 + 40) + 4 * U * span
    both = 2 * e + 8 * U * (1 + float((y.max(1).values - y.min(1).values).max()) / T)
    off = 2.0 ** -8 * p.scatter(1, at, 0.0) * g.abs() + both * (p + full) * g.abs()
    for name, got, want, tol in (("d_rho", d_rho, d @ b, off @ b.abs()), ("d_w", d_w, d.T @ a, off.T @ a.abs())):
        tol = tol + 2.0 ** -8 * want.abs() + 1e-30
        bad = (got.double() - want).abs() > tol
        assert not bad.any(), (name, int(bad.sum()), float((got.double() - want).norm() / want.norm()))
