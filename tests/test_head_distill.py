"""dls_head_distill against a float64 computation on the same bf16 states and weights, and its gradients against
differences of the loss: ranks from 8 to 256 (those that fill a matrix tile and those that do not), one row and many,
vocabularies that end inside a tile, one to 256 teacher entries, repeated ids, tokens that all rows share, positions
left out, logits far from 0.

Tolerances: a logit sums r exact products in float32, within u r |rho|.|W| (u = 2^-24); lse and loss then follow
test_distill.py with V / 256 replaced by the additions of one lane, V / 32 at most.  The gradients sum
d_v W_v with every probability rounded to bf16 (8 significant bits, 2^-9 relative on average at most 2^-8) and are
rounded to bf16 once: entry by entry within 2^-8 (sum |p_v W_v| |g / T| M + |result|) plus float32's share, bounded by
the same sum times 2^-12 (its lse, its logits and its additions are good to 1e-5 of a probability each).
"""
import math

import numpy as np
import pytest
import torch

from paper_2607_07409_amd import binding as B

U = 2.0 ** -24
BF16 = torch.bfloat16


def _make(rows, V, r, K, seed, std=3.0, renorm=True, ragged=False):
    g = torch.Generator().manual_seed(seed)
    rho = torch.randn((rows, r), generator=g).to(BF16)
    w = (torch.randn((V, r), generator=g) * (std / math.sqrt(r))).to(BF16)
    ids = (torch.rand((rows, K), generator=g) ** 3 * V).int().clamp(max=V - 1)   # repeats, low ids often
    y = torch.randn((rows, K), generator=g) * 2
    if not renorm:
        y = torch.log_softmax(y, 1) - 0.1
    if ragged:
        kind = torch.rand((rows, K), generator=g)
        ids[kind < 0.15], ids[(kind > 0.15) & (kind < 0.25)], y[(kind > 0.25) & (kind < 0.3)] = -1, V, -math.inf
        ids[0] = -1
    weight = torch.randn(rows, generator=g)
    return rho.cuda(), w.cuda(), ids.cuda(), y.cuda(), weight.cuda()


def _reference(rho, w, ids, y, weight, T, renorm):
    """Float64 on the GPU, by the formulas; also the sums that bound the rounding."""
    V = w.shape[0]
    x, rho, w = (rho.double() @ w.double().T) / T, rho.double(), w.double()
    there = (ids >= 0) & (ids < V) & (y > -math.inf)
    y = y.double().masked_fill(~there, -math.inf)
    if renorm:
        q = torch.softmax(y / T, 1).masked_fill(~there, 0.0).nan_to_num(0.0)
    else:
        q = y.exp()
    at = ids.long().clamp(0, V - 1)
    lse = torch.logsumexp(x, 1)
    logp = x.gather(1, at) - lse[:, None]
    loss = torch.where(q > 0, q * (q.clamp(min=1e-300).log() - logp), 0.0).sum(1)
    g = (weight.double() if weight is not None else torch.ones_like(lse)) / T
    p = (x - lse[:, None]).exp() * (q.sum(1) * g)[:, None]
    d = p.scatter_add(1, at, -q * g[:, None])
    return dict(loss=loss, lse=lse, d_rho=d @ w, d_w=d.T @ rho, rho_sum=p.abs() @ w.abs(), w_sum=p.abs().T @ rho.abs(),
                rho_q=(q * g.abs()[:, None]).sum(1)[:, None] * w.abs().max(), mass=q.sum(1), top=x.abs().max(),
                size=(rho.norm(dim=1).max() * w.norm(dim=1).max()).item() / T, span=(logp.abs() * (q > 0)).max())


def _check(rho, w, ids, y, weight, T, renorm, got):
    loss, lse, d_rho, d_w = got
    ref = _reference(rho, w, ids, y, weight, T, renorm)
    V, r = w.shape
    e = U * (V / 32 + 40) + 4 * U * float(ref["top"]) + U * r * ref["size"]
    assert ((lse.double() - ref["lse"]).abs() <= e + 2 * U * ref["lse"].abs()).all()
    assert ((loss.double() - ref["loss"]).abs() <= ref["mass"] * (2 * e) + 64 * U * (1 + float(ref["span"])) + 4 * U * ref["loss"].abs()).all()
    if d_rho is None:
        return ref
    for name, out, bound in (("d_rho", d_rho, ref["rho_sum"]), ("d_w", d_w, ref["w_sum"])):
        want = ref[name]
        tol = (2.0 ** -8 + 2.0 ** -12) * bound + 2.0 ** -8 * want.abs() + 2.0 ** -20 * (ref["rho_q"] if name == "d_rho" else want.abs().max()) + 1e-30
        bad = (out.double() - want).abs() > tol
        assert not bad.any(), (name, bad.sum().item(), torch.nonzero(bad)[:4].tolist(), out[bad][:4], want[bad][:4], tol[bad][:4])
        # and as a whole no further off than the two roundings to bf16 allow
        assert (out.double() - want).norm() <= 2.0 ** -8 * (want.norm() + 0.5 * bound.norm()) + 1e-30
    return ref


@pytest.mark.gpu
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("rows,V,r,K", [(1, 1, 8, 1), (1, 33, 16, 3), (3, 1000, 32, 5), (65, 257, 40, 16), (64, 4096, 64, 20), (31, 2049, 72, 256),
                                        (100, 5003, 128, 64), (257, 3001, 136, 33), (16, 32003, 256, 64), (300, 10007, 256, 20), (700, 1031, 200, 50)])
def test_matches_float64(rows, V, r, K, renorm):
    rho, w, ids, y, weight = _make(rows, V, r, K, rows + V + r, renorm=renorm)
    T = 1.0 if renorm else 2.0
    got = B.head_distill(rho, w, ids, y, grad_loss=weight, temperature=T, renormalise=renorm, want_grads=True)
    _check(rho, w, ids, y, weight, T, renorm, got)
    loss, lse, none, none2 = B.head_distill(rho, w, ids, y, temperature=T, renormalise=renorm)
    assert none is None and none2 is None
    _check(rho, w, ids, y, None, T, renorm, (loss, lse, None, None))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V,r", [(2100, 600, 256), (1500, 513, 64), (4097, 2000, 128)])
def test_tiles_of_w_shared_by_workgroups(rows, V, r):
    """Fewer tiles of W than CUs and many rows: the rows are split and the parts joined."""
    rho, w, ids, y, weight = _make(rows, V, r, 24, rows, ragged=True)
    _check(rho, w, ids, y, weight, 1.0, True, B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True))


@pytest.mark.gpu
def test_the_main_vocabulary():
    rho, w, ids, y, weight = _make(40, 151936, 256, 64, 5)
    _check(rho, w, ids, y, weight, 1.0, True, B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True))


@pytest.mark.gpu
@pytest.mark.parametrize("renorm", [True, False])
def test_absent_entries_and_positions_left_out(renorm):
    rho, w, ids, y, _ = _make(130, 3001, 128, 20, 9, renorm=renorm, ragged=True)
    loss, lse, d_rho, d_w = got = B.head_distill(rho, w, ids, y, temperature=0.7, renormalise=renorm, want_grads=True)
    _check(rho, w, ids, y, None, 0.7, renorm, got)
    assert loss[0] == 0 and not d_rho[0].any()
    none = B.head_distill(rho, w, torch.full_like(ids, -1), y, want_grads=True)
    assert not none[0].any() and not none[2].any() and not none[3].any() and torch.isfinite(none[1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("r", [64, 128, 256])
def test_one_token_of_all_rows(r):
    """Every entry of every row names one token: one list holds them all."""
    rho, w, ids, y, weight = _make(500, 1500, r, 40, 11)
    ids.fill_(777)
    _check(rho, w, ids, y, weight, 1.0, True, B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True))


@pytest.mark.gpu
@pytest.mark.parametrize("r", [64, 128, 256])
def test_references_that_rise(r):
    """Logits that grow along the vocabulary by hundreds, so the running reference moves again and again."""
    rho, w, ids, y, weight = _make(70, 4099, r, 16, 13)
    direction = torch.sign(rho[0].float())
    rho.copy_((rho.float().abs() * direction).to(BF16))
    ramp = torch.linspace(-1.0, 1.0, 4099, device="cuda")[:, None] * direction * (300.0 / r)
    w.copy_((w.float() + ramp).to(BF16))
    _check(rho, w, ids, y, weight, 1.0, True, B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True))
    w2 = w.flip(0).contiguous()
    _check(rho, w2, ids, y, weight, 1.0, True, B.head_distill(rho, w2, ids, y, grad_loss=weight, want_grads=True))


@pytest.mark.gpu
def test_far_from_zero():
    """Logits near -400 everywhere: a probability's exponent is relative to the row's own largest logit."""
    rho, w, ids, y, weight = _make(40, 2000, 64, 8, 17, std=1.0)
    rho[:, 0], w[:, 0] = 20.0, -20.0
    _check(rho, w, ids, y, weight, 1.0, True, B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True))


@pytest.mark.gpu
def test_gradients_against_differences():
    """Directions along single states and weights, steps that bf16 holds exactly.  h = 2^-4 of values near 1:
    h^2 / 6 |f'''| <= 1e-3 of the logit scale, float32 losses leave 1e-6 / h, bf16 gradients 2^-7 of the sums."""
    rows, V, r, K = 4, 24, 16, 5
    g = torch.Generator().manual_seed(3)
    quarter = lambda shape: (torch.randint(-8, 9, shape, generator=g) / 8.0)   # noqa: E731  (exact with a step of 1/16)
    rho, w = quarter((rows, r)), quarter((V, r))
    ids = torch.randint(0, V, (rows, K), generator=g, dtype=torch.int32).cuda()
    y = torch.randn((rows, K), generator=g).cuda()
    total = lambda a, b: B.head_distill(a.to(BF16).cuda(), b.to(BF16).cuda(), ids, y)[0].double().sum().item()   # noqa: E731
    _, _, d_rho, d_w = B.head_distill(rho.to(BF16).cuda(), w.to(BF16).cuda(), ids, y, want_grads=True)
    h = 1.0 / 16
    for k in range(12):
        a, b = k % rows, (5 * k) % r
        up, down = rho.clone(), rho.clone()
        up[a, b] += h
        down[a, b] -= h
        assert abs((total(up, w) - total(down, w)) / (2 * h) - d_rho[a, b].item()) < 1e-2
        a = (7 * k) % V
        up, down = w.clone(), w.clone()
        up[a, b] += h
        down[a, b] -= h
        assert abs((total(rho, up) - total(rho, down)) / (2 * h) - d_w[a, b].item()) < 1e-2


@pytest.mark.gpu
def test_agrees_with_stored_logits():
    """distill_loss on the same logits, stored in float32."""
    rho, w, ids, y, _ = _make(50, 5003, 128, 20, 21)
    x = (rho.double() @ w.double().T).float()
    loss, lse, _ = B.distill_loss(x, ids, y, temperature=2.0)
    got = B.head_distill(rho, w, ids, y, temperature=2.0)
    assert (loss - got[0]).abs().max() < 2e-5 and (lse - got[1]).abs().max() < 2e-5


@pytest.mark.gpu
def test_same_bits_on_another_stream_and_in_a_graph():
    rho, w, ids, y, weight = _make(90, 5003, 128, 40, 23)
    want = B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    many = [B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True, stream=st) for _ in range(6)]
    st.synchronize()
    for got in many:
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    out = tuple(torch.empty_like(t) for t in want)
    ws = torch.empty(B.head_distill_workspace_size(90, 5003, 128, 40), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.head_distill(rho, w, ids, y, grad_loss=weight, out=out, workspace=ws)
    for seed in (24, 25, 26):
        new = _make(90, 5003, 128, 40, seed)
        for old, t in zip((rho, w, ids, y, weight), new):
            old.copy_(t)
        want = B.head_distill(rho, w, ids, y, grad_loss=weight, want_grads=True)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))


@pytest.mark.gpu
def test_no_rows():
    rho, w, ids, y, _ = _make(2, 100, 64, 4, 27)
    loss, lse, d_rho, d_w = B.head_distill(rho[:0], w, ids[:0], y[:0], want_grads=True)
    assert loss.shape == (0,) and d_rho.shape == (0, 64) and not d_w.any()
    assert B.head_distill(rho[:0], w, ids[:0], y[:0])[0].shape == (0,)


@pytest.mark.gpu
def test_binding_refuses():
    rho, w, ids, y, weight = _make(4, 100, 64, 4, 29)
    for bad in ((rho.float(), w, ids, y), (rho, w.float(), ids, y), (rho, w, ids.long(), y), (rho, w, ids, y.double())):
        with pytest.raises(TypeError):
            B.head_distill(*bad)
    for bad in ((rho[0], w, ids, y), (rho, w[:, :32], ids, y), (rho, w, ids[:3], y), (rho[:, ::2], w[:, ::2], ids, y), (rho.cpu(), w, ids, y),
                (rho, w.cpu(), ids, y)):
        with pytest.raises(ValueError):
            B.head_distill(*bad)
    with pytest.raises(ValueError):
        B.head_distill(rho, w, ids, y, grad_loss=weight[:2], want_grads=True)
    for kw in (dict(temperature=0.0), dict(temperature=math.nan), dict(out=(None, None, None, None)),
               dict(out=(None, None, torch.empty_like(rho), None)), dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(B.DlsError):
            B.head_distill(rho, w, ids, y, **kw)
    with pytest.raises(B.DlsError):
        B.head_distill(rho[:, :4].contiguous(), w[:, :4].contiguous(), ids, y)


# ------------------------------------------------------------------------------------------------
# host side (no GPU): refusals of the C entry point before any device call
# ------------------------------------------------------------------------------------------------
PTR = 0x7f0000000000


def _call(rho=PTR, w=PTR, rows=4, V=1000, r=64, ids=PTR, values=PTR, k=5, flags=0, T=1.0, reserved=0, weight=PTR, loss=PTR, lse=PTR, d_rho=PTR,
          d_w=PTR, ws=PTR, wsb=1 << 34):
    te = B.Teacher(ids, values, k, flags, T, reserved)
    return B.lib().dls_head_distill(rho, w, rows, V, r, te, weight, loss, lse, d_rho, d_w, ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), 2), (dict(rows=(1 << 20) + 1), 2), (dict(V=0), 2), (dict(V=(1 << 20) + 1), 2), (dict(r=0), 2), (dict(r=12), 2), (dict(r=264), 2),
    (dict(k=0), 2), (dict(k=257), 2), (dict(flags=4), 1), (dict(reserved=1), 1), (dict(T=0.0), 1), (dict(T=math.nan), 1), (dict(rho=None), 1),
    (dict(w=None), 1), (dict(ids=None), 1), (dict(values=None), 1), (dict(d_rho=None), 1), (dict(d_w=None), 1), (dict(rho=PTR + 8), 1),
    (dict(w=PTR + 8), 1), (dict(d_rho=PTR + 8), 1), (dict(d_w=PTR + 8), 1), (dict(loss=PTR + 2), 1), (dict(weight=PTR + 2), 1), (dict(ws=None), 1),
    (dict(ws=PTR + 16), 1), (dict(wsb=100), 4), (dict(loss=None, lse=None, d_rho=None, d_w=None), 1)])
def test_entry_point_refuses(kw, status):
    assert _call(**kw) == status
    assert B.lib().dls_last_error()


def test_sizes():
    assert _call(rows=0, rho=None, ids=None, d_rho=None, d_w=None) == 0
    assert B.head_distill_workspace_size(0, 1000, 64, 5) == 0 and B.head_distill_workspace_size(4, 1000, 60, 5) == 0
    assert 0 < B.head_distill_workspace_size(4, 1000, 64, 5, False) < B.head_distill_workspace_size(4, 1000, 64, 5, True)
    assert B.head_distill_workspace_size(1 << 20, 1 << 20, 256, 256) < 1 << 33
