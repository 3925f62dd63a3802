"""Rows of logits that hold a NaN or +inf, as a diverged training step gives them: such a row's loss, log-sum-exp, statistics and
whole gradient are NaN, by every kernel that may take the call, and the rows beside it are as they are without it."""
import math

import pytest
import torch

from paper_2607_07409_amd import binding as B

BF16, F32 = torch.bfloat16, torch.float32
BITS = {"nan": {BF16: 0x7FC0, F32: 0x7FC00000}, "nan with the sign": {BF16: -1, F32: -1}, "inf": {BF16: 0x7F80, F32: 0x7F800000}}


def _spoil(x, row, where, what):
    places = {"first": 0, "inside": x.shape[1] // 2 + 3, "last": x.shape[1] - 1, "all": slice(None)}[where]
    x.view(torch.int16 if x.dtype == BF16 else torch.int32)[row, places] = BITS[what][x.dtype]


def _logits(rows, V, dtype, seed):
    return (3 * torch.randn((rows, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))).to(dtype)


WHERE = ["first", "inside", "last", "all"]


def _same(a, b, rows):
    return all(torch.equal(a[r], b[r]) for r in rows)


# (rows, V, type): whole rows by 256 and by 1,024 threads, rows read twice, parts of rows, rows that start at every alignment
SHAPES = [(3, 33, F32), (5, 5003, BF16), (5, 5003, F32), (600, 5003, BF16), (4, 100003, BF16), (70, 100003, BF16), (3, 90001, F32),
          (1100, 1001, F32)]


@pytest.mark.gpu
@pytest.mark.parametrize("what", list(BITS))
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("rows,V,dtype", SHAPES)
def test_distillation(rows, V, dtype, where, what):
    K, g = 9, torch.Generator().manual_seed(V)
    x = _logits(rows, V, dtype, rows)
    ids = torch.randint(1, V - 1, (rows, K), generator=g, dtype=torch.int32).cuda()
    ids[ids == V // 2 + 3] = 1   # no entry names the spoilt place
    y = torch.randn((rows, K), generator=g).cuda()
    w = (0.5 + torch.rand(rows, generator=g)).cuda()
    clean = B.distill_loss(x, ids, y, grad_loss=w, want_grad=True)
    clean_alone = B.distill_grad(x, clean[1], ids, y, grad_loss=w)
    _spoil(x, 1, where, what)
    others = [r for r in (0, 2, 3, rows - 1) if r < rows and r != 1]
    loss, lse, grad = B.distill_loss(x, ids, y, grad_loss=w, want_grad=True)
    alone = B.distill_grad(x, lse, ids, y, grad_loss=w)
    loss2, lse2, _ = B.distill_loss(x, ids, y)
    for t in (loss, lse, grad, alone, loss2, lse2):
        assert torch.isnan(t[1].float()).all(), (t.shape, t[1])
    assert all(_same(a, b, others) for a, b in ((loss, clean[0]), (lse, clean[1]), (grad, clean[2]), (alone, clean_alone)))
    # a position that the loss leaves out is 0 whatever the logits
    ids[1] = -1
    loss, lse, grad = B.distill_loss(x, ids, y, grad_loss=w, want_grad=True)
    alone = B.distill_grad(x, lse, ids, y, grad_loss=w)
    assert loss[1] == 0 and math.isnan(lse[1]) and not grad[1].any() and not alone[1].any()


@pytest.mark.gpu
@pytest.mark.parametrize("what", list(BITS))
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("k", [0, 20])
@pytest.mark.parametrize("rows,V,dtype", [(3, 33, BF16), (5, 5003, BF16), (5, 5003, F32), (1025, 5003, BF16), (1025, 20011, BF16), (4, 100003, BF16)])
def test_log_probabilities(rows, V, dtype, k, where, what):
    x = _logits(rows, V, dtype, rows)
    tok = (torch.arange(rows, dtype=torch.int32, device="cuda") * 7 + 1) % V
    clean = B.token_logprobs(x, tok, top_k=k)
    _spoil(x, 1, where, what)
    stats, ids, logps = B.token_logprobs(x, tok, top_k=k)
    assert torch.isnan(stats[1]).all(), stats[1]
    there = ids[1] >= 0
    assert torch.isnan(logps[1][there]).all() and (logps[1][~there] == -math.inf).all()
    # the alternatives are still the numbers in their order
    s = x[1].float()
    order = torch.sort(s.masked_fill(torch.isnan(s), -math.inf), descending=True, stable=True)
    want = torch.where(order.values > -math.inf, order.indices, -1)[:k]
    assert torch.equal(ids[1, :len(want)], want.int()) and (ids[1, len(want):] == -1).all()
    others = [r for r in (0, 2, 3, rows - 1) if r < rows and r != 1]
    assert all(_same(a, b, others) for a, b in zip((stats, ids, logps), clean))


@pytest.mark.gpu
@pytest.mark.parametrize("renorm,value", [(True, math.nan), (True, math.inf), (False, math.nan)])
@pytest.mark.parametrize("rows,V,dtype", [(5, 5003, BF16), (600, 5003, F32), (4, 100003, BF16)])
def test_a_teacher_that_is_not_a_number(rows, V, dtype, renorm, value):
    """One value of a row's entries (its id inside the vocabulary): loss and gradient of that row are NaN, the others' as they are."""
    K, g = 9, torch.Generator().manual_seed(V)
    x = _logits(rows, V, dtype, rows)
    ids = torch.randint(0, V, (rows, K), generator=g, dtype=torch.int32).cuda()
    y = torch.log_softmax(torch.randn((rows, K), generator=g), 1).cuda()
    clean = B.distill_loss(x, ids, y, renormalise=renorm, want_grad=True)
    y[1, 4] = value
    loss, lse, grad = B.distill_loss(x, ids, y, renormalise=renorm, want_grad=True)
    alone = B.distill_grad(x, lse, ids, y, renormalise=renorm)
    assert math.isnan(loss[1]) and torch.isnan(grad[1]).all() and torch.isnan(alone[1]).all()
    others = [0, 2, 3, rows - 1]
    assert torch.equal(lse, clean[1]) and _same(loss, clean[0], others) and _same(grad, clean[2], others)
    rho, w = _logits(rows, 64, BF16, 1), _logits(997, 64, BF16, 2) / 8
    ids %= 997
    clean = B.head_distill(rho, w, ids, torch.where(torch.isfinite(y), y, 0.0), renormalise=renorm, want_grads=True)
    loss, lse, d_rho, d_w = B.head_distill(rho, w, ids, y, renormalise=renorm, want_grads=True)
    assert math.isnan(loss[1]) and torch.isnan(d_rho[1]).all() and torch.isnan(d_w).all()
    assert torch.equal(lse, clean[1]) and _same(loss, clean[0], others) and _same(d_rho, clean[2], others)
    # outside the vocabulary it is absent
    ids[1, 4] = 997
    assert torch.isfinite(B.head_distill(rho, w, ids, y, renormalise=renorm)[0]).all()
