"""A call that asks for gradients and gives `out` without a place for them is refused."""
import pytest
import torch

from paper_2607_07409_amd import binding as B


@pytest.mark.gpu
def test_wanted_gradients_need_a_place():
    x = torch.randn((4, 64), device="cuda")
    ids, y = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    loss, lse = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    with pytest.raises(ValueError, match="gradient"):
        B.distill_loss(x, ids, y, want_grad=True, out=(loss, lse, None))
    grad = torch.empty_like(x)
    assert B.distill_loss(x, ids, y, want_grad=True, out=(loss, lse, grad))[2] is grad
    rho, w = torch.randn((4, 64), device="cuda").bfloat16(), torch.randn((64, 64), device="cuda").bfloat16()
    d_rho, d_w = torch.empty_like(rho), torch.empty_like(w)
    for out in ((loss, lse, None, None), (loss, lse, d_rho, None), (loss, lse, None, d_w)):
        with pytest.raises(ValueError, match="gradient"):
            B.head_distill(rho, w, ids, y, want_grads=True, out=out)
    assert B.head_distill(rho, w, ids, y, want_grads=True, out=(loss, lse, d_rho, d_w))[3] is d_w
