"""dls_distill_loss and dls_distill_grad against the float64 oracle and against differences of the loss: both teacher
forms, both types, split and whole rows, one to 256 teacher entries, repeated, absent and missing ones, slices at every
alignment, gradients in place of the logits, masked rows, rows without any entry and of the type's lowest value.

Tolerances (u = 2^-24): the log-sum-exp is within e = u (V / 256 + 40) + 4 u |s / T|max + 4 u span / T (see
test_token_logprobs), each q within 8 u (1 + span of the values) relative, so the loss is within
M e + 8 u (1 + span) (loss + |log p| + |log q|).  A gradient entry is within |g / T| (p e' + q 8 u (1 + span)) with
e' = 2 e + 4 u, and rounds once to its type (2^-8 or u of it, at least the type's smallest step); a probability below 2^-126 counts as 0.
"""
import math

import numpy as np
import pytest
import torch

from oracle import dels_oracle as O
from paper_2607_07409_amd import binding as B

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
ROUND = {BF16: 2.0 ** -8, F32: U}


def _e(x, T):
    fin = x[np.isfinite(x) & (np.abs(x) < 1e30)]
    top = np.max(np.abs(fin), initial=0.0) / T
    span = min((fin.max() - fin.min()) / T, 200.0) if len(fin) else 0.0
    return U * (len(x) / 256 + 40) + 4 * U * top + 4 * U * span


def _check(logits, ids, values, weight, T, renorm, loss=None, lse=None, grad=None, rows=None):
    x, ids, values = logits.float().cpu().numpy().astype(np.float64), ids.cpu().numpy(), values.cpu().numpy().astype(np.float64)
    w = np.ones(len(x)) if weight is None else weight.cpu().numpy().astype(np.float64)
    loss, lse = (None if t is None else t.cpu().numpy() for t in (loss, lse))
    out = None if grad is None else grad.float().cpu().numpy().astype(np.float64)
    for r in range(len(x)) if rows is None else rows:
        want, want_lse, want_grad = O.distill_row(x[r], ids[r], values[r], w[r], T, renorm)
        q = O.teacher_weights(ids[r], values[r], x.shape[1], T, renorm)
        e, mass = _e(x[r], T), q.sum()
        y = values[r][q > 0]
        span = ((y.max() - y.min()) / (T if renorm else 1.0) + (0.0 if renorm else np.abs(y).max())) if len(y) else 0.0
        teach = 8 * U * (1 + span)
        if loss is not None:
            if math.isfinite(want):
                assert abs(loss[r] - want) <= mass * e + teach * (abs(want) + 2 * span + 20) * max(mass, 1e-30) + 4 * U * abs(want), (r, loss[r], want)
            else:
                assert loss[r] == want
        if lse is not None and not -math.inf < want_lse < -1e37:
            if math.isfinite(want_lse):
                assert abs(lse[r] - want_lse) <= e + 2 * U * abs(want_lse), (r, lse[r], want_lse)
            else:
                assert lse[r] == want_lse
        if out is not None:
            qv = np.zeros(x.shape[1])
            np.add.at(qv, ids[r][q > 0], q[q > 0])
            p_part = want_grad * (T / w[r]) + qv if w[r] else qv
            tol = abs(w[r] / T) * (np.abs(p_part) * (2 * e + 4 * U) + qv * teach) + ROUND[grad.dtype] * 1.01 * np.abs(want_grad) + 1.01 * 2.0 ** -126 * (1 + abs(w[r] / T))
            bad = np.abs(out[r] - want_grad) > tol
            assert not bad.any(), (r, np.flatnonzero(bad)[:5], out[r][bad][:5], want_grad[bad][:5])


def _student(rows, V, dtype, seed, pad=0, offset=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, V + pad + offset), generator=g) * 3).to(dtype).cuda()[:, offset:offset + V]


def _teacher(rows, V, K, seed, renorm=True, ragged=False):
    """Ids drawn with repeats, some outside [0, V); values or log probabilities."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, V, (rows, K), generator=g, dtype=torch.int32)
    y = torch.randn((rows, K), generator=g) * 3
    if not renorm:
        y = torch.log_softmax(y, 1) - 0.2
    if ragged:
        kind = torch.rand((rows, K), generator=g)
        ids[kind < 0.1] = -1
        ids[(kind > 0.1) & (kind < 0.2)] = V
        ids[(kind > 0.2) & (kind < 0.25)] = 2**31 - 1
        y[(kind > 0.25) & (kind < 0.35)] = -math.inf
        ids[0] = -5        # a row without entries
    return ids.cuda(), y.cuda()


def _weight(rows, seed):
    w = torch.randn(rows, generator=torch.Generator().manual_seed(seed))
    w[-1] = 0.0
    return w.cuda()


def _all(x, ids, y, w, T, renorm, rows=None):
    loss, lse, none = B.distill_loss(x, ids, y, temperature=T, renormalise=renorm)
    assert none is None
    _check(x, ids, y, None, T, renorm, loss=loss, lse=lse, rows=rows)
    loss2, lse2, grad = B.distill_loss(x, ids, y, grad_loss=w, temperature=T, renormalise=renorm, want_grad=True)
    _check(x, ids, y, w, T, renorm, loss=loss2, lse=lse2, grad=grad, rows=rows)
    alone = B.distill_grad(x, lse, ids, y, grad_loss=w, temperature=T, renormalise=renorm)
    _check(x, ids, y, w, T, renorm, grad=alone, rows=rows)
    return loss, lse, grad, alone


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("rows,V,K", [(1, 1, 1), (2, 2, 5), (3, 9, 16), (2, 1003, 256), (5, 5003, 20), (3, 32003, 100), (2, 151936, 64)])
def test_matches_oracle(rows, V, K, renorm, dtype):
    x, (ids, y) = _student(rows, V, dtype, V + K), _teacher(rows, V, K, K, renorm)
    _all(x, ids, y, _weight(rows, V), 1.0, renorm)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("renorm", [True, False])
def test_whole_rows(renorm, dtype):
    x, (ids, y) = _student(1025, 5003, dtype, 3), _teacher(1025, 5003, 40, 4, renorm, ragged=True)
    _all(x, ids, y, _weight(1025, 5), 2.0, renorm, rows=[0, 1, 2, 511, 1023, 1024])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [0.1, 0.7, 4.0])
def test_temperature_and_absent_entries(T, dtype):
    for renorm in (True, False):
        x, (ids, y) = _student(6, 7001, dtype, 13), _teacher(6, 7001, 33, 14, renorm, ragged=True)
        loss, _, grad, alone = _all(x, ids, y, _weight(6, 15), T, renorm)
        assert loss[0] == 0 and not grad[0].any() and not alone[0].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset", range(9))
def test_slices_at_any_alignment(offset, dtype):
    """Logits at one alignment, gradients at another, both inside wider rows whose other entries stay."""
    V, (ids, y) = 4099, _teacher(4, 4099, 20, 24)
    x, w = _student(4, V, dtype, 21 + offset, pad=offset % 4, offset=offset), _weight(4, 25)
    wide = torch.full((4, V + 13), 7.0, dtype=dtype, device="cuda")
    grad = wide[:, 5:5 + V]
    loss, lse, got = B.distill_loss(x, ids, y, grad_loss=w, out=(torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), grad))
    assert got is grad
    _check(x, ids, y, w, 1.0, True, loss=loss, lse=lse, grad=grad)
    assert (wide[:, :5] == 7).all() and (wide[:, 5 + V:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,V", [(3, 32003), (1024, 4099)])
def test_gradient_in_place(rows, V, dtype):
    x, (ids, y), w = _student(rows, V, dtype, 31, pad=3, offset=2), _teacher(rows, V, 64, 32), _weight(rows, 33)
    want = B.distill_loss(x, ids, y, grad_loss=w, want_grad=True)
    alone = B.distill_grad(x, want[1], ids, y, grad_loss=w)
    for fused in (True, False):
        buf = torch.full((rows, V + 5), 7.0, dtype=dtype, device="cuda")
        s = buf[:, 2:2 + V]
        s.copy_(x)
        if fused:
            B.distill_loss(s, ids, y, grad_loss=w, out=(None, None, s))
        else:
            B.distill_grad(s, want[1], ids, y, grad_loss=w, out=s)
        assert torch.equal(s, want[2] if fused else alone)
        assert (buf[:, :2] == 7).all() and (buf[:, 2 + V:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V,dtype", [(64, 100003, BF16), (65, 100003, BF16), (64, 99999, BF16), (65, 81919, F32), (513, 24571, BF16), (513, 24577, BF16), (513, 12287, F32)])
def test_where_the_choice_of_kernel_changes(rows, V, dtype):
    """Numbers of rows and lengths at which another kernel or workgroup takes over, also with the gradient in place."""
    x, (ids, y), w = _student(rows, V, dtype, 41, pad=1), _teacher(rows, V, 30, 42, ragged=True), _weight(rows, 43)
    grad = _all(x, ids, y, w, 1.0, True, rows=[0, 1, rows // 2, rows - 1])[2]
    s = torch.empty((rows, V + 1), dtype=dtype, device="cuda")[:, :V].copy_(x)
    loss, lse, _ = B.distill_loss(s, ids, y, grad_loss=w, out=(torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), s))
    _check(x, ids, y, w, 1.0, True, loss=loss, lse=lse, grad=s, rows=[0, 1, rows // 2, rows - 1])
    assert torch.equal(s, grad)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("whole", [False, True])
def test_special_rows(whole, dtype):
    V, g, low = 3001, np.random.default_rng(7), torch.finfo(dtype).min
    x = np.stack([np.full(V, -np.inf), np.full(V, low), np.where(g.random(V) < 0.9, -np.inf, g.normal(0, 3, V)),
                  np.where(g.random(V) < 0.9, low, g.normal(0, 3, V)), np.full(V, 1.25), g.normal(0, 3, V) + 1e4,
                  np.where(np.arange(V) == 17, 90.0, g.normal(0, 1, V)), g.normal(0, 3, V)]).astype(np.float32)
    n = len(x)
    if whole:
        x = np.tile(x, (128, 1))
    x = torch.from_numpy(x).to(dtype).cuda()
    ids, y = _teacher(len(x), V, 8, 42)
    for r in (2, 3):   # entries that the mask leaves
        keep = torch.nonzero(x[r] > -1e30)[:, 0][:8].int()
        ids[r] = keep
    ids[6] = 17
    ids[7], y[7] = 5, -math.inf    # no entry
    w = _weight(len(x), 43)
    loss, lse, grad, alone = _all(x, ids, y, w, 1.0, True, rows=[r for r in range(n) if r not in (0, 1)])
    # nothing to choose from: the loss has no finite value, the gradient is the teacher's part alone
    assert loss[0] == math.inf and lse[0] == -math.inf
    _check(x, ids, y, w, 1.0, True, loss=loss, lse=lse, grad=grad, rows=[0, 1])
    _check(x, ids, y, w, 1.0, True, grad=alone, rows=[0])
    assert torch.isfinite(alone[1].float()).all()   # a float32 log-sum-exp of -1e38 holds no log V
    # a masked entry that the teacher wants
    ids[2, 0] = int(torch.nonzero(x[2] == -math.inf)[0])
    y[2] = 0.0
    loss, _, grad = B.distill_loss(x, ids, y, grad_loss=w, want_grad=True)
    assert loss[2] == math.inf and torch.isfinite(grad[2].float()).all()
    _check(x, ids, y, w, 1.0, True, grad=grad, rows=[2])


@pytest.mark.gpu
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_gradient_against_differences(T, renorm):
    """Central differences of the loss, a row for each step up and down: h = 0.02 leaves h^2 / 6 |f'''| <= 7e-5 / T^3
    and float32 losses of at most 8 leave 2 x 2e-6 / 2h = 1e-4."""
    V, h = 24, 0.02
    x, (ids, y) = _student(1, V, F32, 51), _teacher(1, V, 6, 52, renorm)
    step = torch.cat([torch.eye(V), -torch.eye(V)]).cuda() * h
    many = (x + step).contiguous()
    loss = B.distill_loss(many, ids.expand(2 * V, -1).contiguous(), y.expand(2 * V, -1).contiguous(), temperature=T,
                          renormalise=renorm)[0].double()
    moved = (many[:V] - many[V:]).double().diagonal()
    grad = B.distill_loss(x, ids, y, temperature=T, renormalise=renorm, want_grad=True)[2][0].double()
    assert ((loss[:V] - loss[V:]) / moved - grad).abs().max() < 2e-4


@pytest.mark.gpu
def test_teacher_entries_from_token_logprobs():
    """A teacher's alternatives are a student's targets: at the teacher's own logits the loss is -M log M + ... of its
    kept mass against itself, and its gradient vanishes outside rounding once every entry is kept."""
    x = _student(4, 200, F32, 61)
    _, ids, lps = B.token_logprobs(x, top_k=200, temperature=2.0)
    loss, _, grad = B.distill_loss(x, ids, lps, temperature=2.0, renormalise=False, want_grad=True)
    assert loss.abs().max() < 1e-5 and grad.abs().max() < 1e-6


@pytest.mark.gpu
def test_another_stream_and_graph_replays():
    x, (ids, y), w = _student(3, 32003, BF16, 71), _teacher(3, 32003, 20, 72), _weight(3, 73)
    want = B.distill_loss(x, ids, y, grad_loss=w, want_grad=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    many = [B.distill_loss(x, ids, y, grad_loss=w, want_grad=True, stream=st) for _ in range(8)]
    st.synchronize()
    for got in many:
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    out = tuple(torch.empty_like(t) for t in want)
    ws = torch.empty(B.distill_workspace_size(3, 32003), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.distill_loss(x, ids, y, grad_loss=w, out=out, workspace=ws)
    for seed in (74, 75, 76):
        x.copy_(_student(3, 32003, BF16, seed))
        want = B.distill_loss(x, ids, y, grad_loss=w, want_grad=True)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    V, stride = 4099, (1 << 31) + 8
    x, (ids, y) = _student(2, V, BF16, 81), _teacher(2, V, 20, 82)
    buf = torch.empty(stride + V, dtype=BF16, device="cuda")
    far = buf.as_strided((2, V), (stride, 1))
    far.copy_(x)
    loss, lse, _ = B.distill_loss(far, ids, y, out=(torch.empty(2, device="cuda"), torch.empty(2, device="cuda"), far))
    _check(x, ids, y, None, 1.0, True, loss=loss, lse=lse, grad=far)


@pytest.mark.gpu
def test_empty_batch():
    x, ids, y = torch.empty((0, 100), device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda"), torch.empty((0, 3), device="cuda")
    loss, lse, grad = B.distill_loss(x, ids, y, want_grad=True)
    assert loss.shape == (0,) and grad.shape == (0, 100)
    assert B.distill_grad(x, lse, ids, y).shape == (0, 100)


@pytest.mark.gpu
def test_binding_refuses():
    x, (ids, y) = _student(4, 64, F32, 91), _teacher(4, 64, 5, 92)
    lse = torch.zeros(4, device="cuda")
    for bad in ((x.double(), ids, y), (x, ids.long(), y), (x, ids, y.double())):
        with pytest.raises(TypeError):
            B.distill_loss(*bad)
    for bad in ((x.t(), ids, y), (x, ids[:3], y), (x, ids, y[:, :4]), (x, ids.cpu(), y), (x, ids[0], y), (x.cpu(), ids, y)):
        with pytest.raises(ValueError):
            B.distill_loss(*bad)
    for kw in (dict(grad_loss=lse[:3]), dict(out=(None, None, x.bfloat16())), dict(out=(None, None, x[:, :60]))):
        with pytest.raises(ValueError):
            B.distill_loss(x, ids, y, **kw)
    with pytest.raises(ValueError):
        B.distill_grad(x, lse[:2], ids, y)
    for T in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(B.DlsError):
            B.distill_loss(x, ids, y, temperature=T)
        with pytest.raises(B.DlsError):
            B.distill_grad(x, lse, ids, y, temperature=T)
    with pytest.raises(B.DlsError):
        B.distill_loss(x, ids.repeat(1, 60), y.repeat(1, 60))   # 300 entries
    with pytest.raises(B.DlsError):
        B.distill_loss(x, ids, y, out=(None, None, None))


# ------------------------------------------------------------------------------------------------
# host side (no GPU): refusals of the C entry points before any device call
# ------------------------------------------------------------------------------------------------
PTR = 0x7f0000000000


def _call(fn="loss", logits=PTR, dtype=1, rows=4, V=1000, stride=1000, ids=PTR, values=PTR, k=5, flags=0, T=1.0, reserved=0,
          weight=PTR, loss=PTR, lse=PTR, grad=PTR + 4096, gstride=1000, ws=PTR, wsb=1 << 30):
    te = B.Teacher(ids, values, k, flags, T, reserved)
    if fn == "loss":
        return B.lib().dls_distill_loss(logits, dtype, rows, V, stride, te, weight, loss, lse, grad, gstride, ws, wsb, None)
    return B.lib().dls_distill_grad(logits, dtype, rows, V, stride, lse, te, weight, grad, gstride, None)


BAD = [(dict(dtype=2), 3), (dict(rows=-1), 2), (dict(rows=(1 << 20) + 1), 2), (dict(V=0), 2), (dict(V=(1 << 24) + 1, stride=1 << 25, gstride=1 << 25), 2),
       (dict(stride=999), 2), (dict(gstride=999), 2), (dict(k=0), 2), (dict(k=257), 2), (dict(flags=2), 1), (dict(reserved=1), 1),
       (dict(T=0.0), 1), (dict(T=math.nan), 1), (dict(T=math.inf), 1), (dict(ids=None), 1), (dict(values=None), 1),
       (dict(ids=PTR + 2), 1), (dict(logits=None), 1), (dict(logits=PTR + 1), 1), (dict(grad=PTR + 1), 1), (dict(weight=PTR + 2), 1),
       (dict(lse=PTR + 2), 1), (dict(grad=PTR, gstride=1008), 1)]


@pytest.mark.parametrize("fn", ["loss", "grad"])
@pytest.mark.parametrize("kw,status", BAD)
def test_entry_points_refuse(fn, kw, status):
    assert _call(fn, **kw) == status
    assert B.lib().dls_last_error()


@pytest.mark.parametrize("fn,kw,status", [("loss", dict(loss=None, lse=None, grad=None), 1), ("loss", dict(loss=PTR + 2), 1),
                                          ("loss", dict(ws=None), 1), ("loss", dict(ws=PTR + 8), 1), ("loss", dict(wsb=8), 4),
                                          ("grad", dict(lse=None), 1), ("grad", dict(grad=None), 1)])
def test_entry_points_refuse_more(fn, kw, status):
    assert _call(fn, **kw) == status


def test_no_rows_and_sizes():
    assert _call(rows=0, logits=None) == 0 and _call("grad", rows=0, logits=None, lse=None) == 0
    assert B.distill_workspace_size(0, 1000) == 0 and B.distill_workspace_size(4, 0) == 0
    assert B.distill_workspace_size(4, 1000) == 4 * 8


def test_teacher_layout():
    import ctypes
    assert ctypes.sizeof(B.Teacher) == 32 and B.Teacher.k.offset == 16 and B.Teacher.temperature.offset == 24
