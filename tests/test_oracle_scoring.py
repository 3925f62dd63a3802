"""Pins of the oracle's scoring and distillation rows (CPU): against torch's float64 log softmax, entropy, stable sort and
automatic differentiation, and by hand where masks leave little or nothing."""
import math

import numpy as np
import pytest
import torch

from oracle import dels_oracle as O


@pytest.mark.parametrize("V,k,T", [(1, 1, 1.0), (7, 3, 0.5), (300, 20, 2.0), (300, 300, 1.0)])
def test_token_logprobs_row(V, k, T):
    g = np.random.default_rng(V + k)
    s = np.round(g.normal(0, 3, V), 1)   # with ties
    logprob, entropy, lse, ids, lps = O.token_logprobs_row(s, V // 2, k, T)
    logp = torch.log_softmax(torch.from_numpy(s) / T, 0)
    assert abs(logprob - logp[V // 2].item()) < 1e-12 and abs(lse - torch.logsumexp(torch.from_numpy(s) / T, 0).item()) < 1e-12
    assert abs(entropy - torch.special.entr(logp.exp()).sum().item()) < 1e-12
    order = torch.sort(torch.from_numpy(s), descending=True, stable=True).indices[:k]
    assert ids.tolist() == order.tolist() and np.allclose(lps, logp[order].numpy(), atol=1e-12)


def test_token_logprobs_row_with_masks():
    inf = math.inf
    logprob, entropy, lse, ids, lps = O.token_logprobs_row([-inf, 2.0, -inf, 2.0], 0, 3)
    assert logprob == -inf and abs(entropy - math.log(2)) < 1e-15 and abs(lse - 2 - math.log(2)) < 1e-15
    assert ids.tolist() == [1, 3, -1] and lps[2] == -inf
    logprob, entropy, lse, ids, lps = O.token_logprobs_row([-inf, -inf], 1, 2)
    assert math.isnan(logprob) and math.isnan(entropy) and lse == -inf and ids.tolist() == [-1, -1]
    low = float(np.finfo(np.float32).min)
    assert abs(O.token_logprobs_row([low] * 4, 2, 1)[0] + math.log(4)) < 1e-12
    assert math.isnan(O.token_logprobs_row([1.0, 2.0], -1, 1)[0]) and math.isnan(O.token_logprobs_row([1.0, 2.0], 2, 1)[0])


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T", [1.0, 2.5])
def test_distill_row(renorm, T):
    g = np.random.default_rng(3)
    V, K, w = 40, 9, 0.7
    s, ids, y = g.normal(0, 2, V), g.integers(0, V, K), g.normal(0, 1, K) - (0 if renorm else 4)
    ids[4] = ids[2]                                # a repeated id
    ids[6], ids[7], y[8] = -1, V, -math.inf        # absent ones
    loss, lse, grad = O.distill_row(s, ids, y, w, T, renorm)
    x = torch.from_numpy(s).requires_grad_()
    there = torch.tensor([0 <= i < V for i in ids]) & torch.from_numpy(y > -math.inf)
    v = torch.from_numpy(y)[there]
    q = torch.softmax(v / T, 0) if renorm else v.exp()
    logp = torch.log_softmax(x / T, 0)[torch.from_numpy(ids)[there]]
    want = (q * (q.log() - logp)).sum()
    (want * w).backward()
    assert abs(loss - want.item()) < 1e-12 and np.allclose(grad, x.grad.numpy(), atol=1e-14)
    assert abs(lse - torch.logsumexp(x / T, 0).item()) < 1e-12


def test_distill_row_with_masks():
    inf = math.inf
    loss, _, grad = O.distill_row([1.0, 2.0], [-1, 5], [0.0, 0.0])
    assert loss == 0 and not grad.any()
    loss, _, grad = O.distill_row([1.0, -inf, 0.0], [1], [0.0])
    assert loss == inf and grad[1] == -1 and abs(grad.sum()) < 1e-15
    loss, lse, grad = O.distill_row([-inf, -inf], [1], [0.0], 2.0)
    assert loss == inf and lse == -inf and grad.tolist() == [0.0, -2.0]
