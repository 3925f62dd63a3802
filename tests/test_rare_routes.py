"""Routes of the scoring and distillation calls that ordinary rows do not take."""
import math

import numpy as np
import pytest
import torch

from paper_2607_07409_amd import binding as B
from test_head_distill import _check as _check_head, _make as _make_head
from test_token_logprobs import _check as _check_logprobs

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,block,most_in_lds", [(BF16, 64, 1024), (F32, 128, 1024)])
@pytest.mark.parametrize("k,blocks", [(8, 24), (40, 60)])
def test_more_candidates_than_the_list_holds(dtype, block, most_in_lds, k, blocks):
    """A row's large entries fill whole blocks, stretches of 64 (float32: 128) entries at V = 60,000: more than k blocks and
    fewer than 2 k + 16, so that all of them are read again, and all of their entries are at or above the bound."""
    V, rows, g = 60000, 1024, np.random.default_rng(5)
    x = g.normal(0, 1, (rows, V)).astype(np.float32)
    assert k < blocks < 2 * k + 16 and blocks * block > most_in_lds
    for r in range(3):
        at = g.permutation(V // block)[:blocks]
        if r == 0:   # side by side
            at = 100 + np.arange(blocks)
        fill = (at[:, None] * block + np.arange(block)).reshape(-1)
        # one value, or float32 ones that agree in their upper half
        x[r, fill] = 50.0 if dtype == BF16 or r == 1 else 50.0 + 0.2 * g.random(len(fill))
        x[r, g.choice(fill, k // 2, replace=False)] = 60.0 + 2.0 * np.arange(k // 2)
    t = torch.from_numpy(x).to(dtype).cuda()
    tok = torch.arange(rows, dtype=torch.int32, device="cuda")
    _check_logprobs(t, tok, k, 1.0, B.token_logprobs(t, tok, top_k=k), rows=[0, 1, 2, 3, rows - 1])


@pytest.mark.gpu
@pytest.mark.parametrize("V", [1 << 20, (1 << 20) - 37])
def test_the_largest_vocabulary_of_a_head(V):
    """As many keys of the entries' sort as there may be, and ids in the last group of the vocabulary."""
    rows, r, K = 5, 24, 40
    rho, w, ids, y, weight = _make_head(rows, V, r, K, 31)
    ids[:, :7] = V - 1 - torch.arange(7, dtype=torch.int32, device="cuda")
    ids[1], ids[2, ::3] = V - 64 + torch.arange(K, dtype=torch.int32, device="cuda") % 64, 0
    ids.clamp_(max=V - 1)
    got = B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True)
    _check_head(rho, w, ids, y, weight, 1.0, True, got)
    loss, _, _, _ = B.head_distill(rho, w, torch.full_like(ids, V), y)
    assert math.isclose(float(loss.abs().max()), 0.0)
