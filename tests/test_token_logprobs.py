"""dls_token_logprobs against the float64 oracle: log probabilities, entropy, log-sum-exp and alternatives over
vocabularies from one entry to 151,936, both types, split and whole rows, slices of wider rows at every alignment,
temperatures, and the rows where such a kernel goes wrong: masked, without any entry, of the type's lowest value,
equal, rising, falling, and one whose few best blocks hold most of its large entries.

Tolerances: a thread sums n = V / 256 positive float32 terms (fewer where rows are split) and the workgroup 40 more
sums, each rounding 2^-24 of the sum; an exponential and its exponent are good to 2^-22 (1 + |x - max| / T); results
round once more.  So lse and log p are within u (n + 40) + 4 u |x / T|max + 4 u |x - max|max / T + 2 u |result|, with
u = 2^-24, and the entropy, whose terms weigh p log p, within 2 (1 + H) times the first.
"""
import math

import numpy as np
import pytest
import torch

from oracle import dels_oracle as O
from paper_2607_07409_amd import binding as B

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def _bounds(x, T):
    """(lse and log p, entropy) tolerances of a row of float64 logits, before their own final rounding."""
    fin = x[np.isfinite(x) & (np.abs(x) < 1e30)]
    top = np.max(np.abs(fin), initial=0.0) / T
    span = (fin.max() - fin.min()) / T if len(fin) else 0.0
    tol = U * (len(x) / 256 + 40) + 4 * U * top + 4 * U * min(span, 200.0)
    return tol, 2 * tol


def _check(logits, tokens, k, T, got, rows=None):
    stats, ids, lps = (t.cpu().numpy() for t in got)
    x = logits.float().cpu().numpy().astype(np.float64)
    tok = [-1] * len(x) if tokens is None else tokens.cpu().tolist()
    for r in range(len(x)) if rows is None else rows:
        logprob, entropy, lse, want_ids, want_lps = O.token_logprobs_row(x[r], tok[r], k, T)
        tol, tol_h = _bounds(x[r], T)
        np.testing.assert_array_equal(ids[r], want_ids, err_msg=f"row {r}")
        for name, got_v, want in (("logprob", stats[r, 0], logprob), ("lse", stats[r, 2], lse)):
            if name == "lse" and -math.inf < want < -1e37:   # only entries beyond the documented magnitude
                assert -math.inf < got_v < -6e37
            elif not math.isfinite(want):
                np.testing.assert_equal(float(got_v), want)
            else:
                assert abs(got_v - want) <= tol + 2 * U * abs(want), (r, got_v, want)
        if math.isnan(entropy):
            assert math.isnan(stats[r, 1])
        else:
            assert abs(stats[r, 1] - entropy) <= tol_h * (1 + entropy), (r, stats[r, 1], entropy)
        fin = np.isfinite(want_lps)
        np.testing.assert_array_equal(np.isfinite(lps[r]), fin)
        assert np.all(np.abs(lps[r][fin] - want_lps[fin]) <= tol + 2 * U * np.abs(want_lps[fin])), r


def _rows(rows, V, dtype, seed, pad=0, offset=0, std=3.0):
    """[rows, V] logits with one raised entry each, a slice of rows of V + pad that starts `offset` entries in."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, V + pad + offset), generator=g) * std
    x[torch.arange(rows), offset + torch.randint(0, V, (rows,), generator=g)] += 9.0
    return x.to(dtype).cuda()[:, offset:offset + V]


def _tokens(rows, V, seed):
    return torch.randint(0, V, (rows,), generator=torch.Generator().manual_seed(seed + 1), dtype=torch.int32).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,V,k", [(1, 1, 1), (3, 2, 5), (5, 7, 3), (2, 255, 256), (4, 2049, 20), (3, 5003, 64), (2, 32003, 128),
                                      (1, 151936, 5), (2, 151936, 256), (1, 151936, 0), (16, 151936, 20)])
def test_matches_oracle(rows, V, k, dtype):
    x, tok = _rows(rows, V, dtype, rows + V), _tokens(rows, V, V)
    _check(x, tok, k, 1.0, B.token_logprobs(x, tok, top_k=k))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [0, 1, 32, 33, 200])
def test_whole_rows(k, dtype):
    """From 1,024 rows on a row is one workgroup's."""
    x, tok = _rows(1025, 5003, dtype, 5), _tokens(1025, 5003, 6)
    _check(x, tok, k, 1.0, B.token_logprobs(x, tok, top_k=k), rows=[0, 1, 7, 512, 1023, 1024])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [0.05, 0.7, 2.0, 50.0])
def test_temperature(T, dtype):
    x, tok = _rows(3, 10007, dtype, 11), _tokens(3, 10007, 12)
    _check(x, tok, 20, T, B.token_logprobs(x, tok, top_k=20, temperature=T))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset", range(9))
def test_slices_at_any_alignment(offset, dtype):
    x, tok = _rows(4, 4099, dtype, 21 + offset, pad=offset % 4, offset=offset), _tokens(4, 4099, 22)
    _check(x, tok, 20, 1.0, B.token_logprobs(x, tok, top_k=20))


def _special(V, dtype):
    g = np.random.default_rng(V)
    low = torch.finfo(dtype).min
    rows = {
        "empty": np.full(V, -np.inf),
        "lowest": np.full(V, low),
        "lowest and -inf": np.where(g.random(V) < 0.5, low, -np.inf),
        "one": np.where(np.arange(V) == V // 2, 1.5, -np.inf),
        "masked": np.where(g.random(V) < 0.97, -np.inf, g.normal(0, 3, V)),
        "masked by the lowest": np.where(g.random(V) < 0.97, low, g.normal(0, 3, V)),
        "equal": np.full(V, -2.0),
        "two values": np.where(g.random(V) < 0.5, 1.0, 2.0),
        "rising": np.linspace(-20, 20, V),
        "falling": np.linspace(20, -20, V),
        "zeros of both signs": np.where(np.arange(V) % 2, 0.0, -0.0),
        "large": g.normal(0, 3, V) + 1e4,
        "sure": np.where(np.arange(V) == V - 1, 80.0, g.normal(0, 1, V)),
    }
    return list(rows), torch.tensor(np.stack(list(rows.values())).astype(np.float32)).to(dtype).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,k", [(9, 4), (3001, 33), (20011, 20)])
@pytest.mark.parametrize("whole", [False, True])
def test_special_rows(V, k, dtype, whole):
    names, x = _special(V, dtype)
    n = len(names)
    if whole:   # as rows of a batch large enough for one workgroup each
        x = x.repeat(-(-1024 // n), 1)
    tok = torch.arange(len(x), dtype=torch.int32, device="cuda") * 7 % V
    tok[3] = V // 2
    _check(x, tok, k, 1.0, B.token_logprobs(x, tok, top_k=k), rows=range(n))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,per", [(BF16, 8), (F32, 4)])
@pytest.mark.parametrize("k", [8, 40])
def test_large_entries_in_few_blocks(dtype, per, k):
    """Seven columns of a thread's chunks hold the large entries, more of them than the candidates' list."""
    V, g = 60000, np.random.default_rng(3)
    x = g.normal(0, 1, (1024, V)).astype(np.float32)
    column = (np.arange(V) // per) % 256
    x[:3, column < 7] += 50.0
    t = torch.from_numpy(x).to(dtype).cuda()
    _check(t, None, k, 1.0, B.token_logprobs(t, top_k=k), rows=[0, 1, 2, 3, 1023])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,V", [(BF16, 263001), (F32, 131101)])
def test_rows_too_long_for_one_workgroup(dtype, V):
    """As many rows as workgroups are wanted, and still parts: a part holds the maxima of 1,024 blocks."""
    x = torch.zeros((1024, V), dtype=dtype, device="cuda")
    x[:3] = _rows(3, V, dtype, 81)
    x[1, V - 1], x[2, 0] = 30.0, 30.0
    tok = _tokens(1024, V, 82)
    _check(x, tok, 20, 1.0, B.token_logprobs(x, tok, top_k=20), rows=[0, 1, 2, 3, 1023])


@pytest.mark.gpu
def test_nan_and_infinite_entries_end():
    """Their results are not specified; ids stay in range and the other rows are untouched."""
    x, tok = _rows(4, 5003, F32, 31), _tokens(4, 5003, 32)
    x[1, 7], x[1, 4000], x[2, 100] = math.nan, math.nan, math.inf
    stats, ids, lps = B.token_logprobs(x, tok, top_k=20)
    assert int(ids.min()) >= -1 and int(ids.max()) < 5003
    assert 7 not in ids[1].tolist() and ids[2, 0].item() == 100
    _check(x, tok, 20, 1.0, (stats, ids, lps), rows=[0, 3])


@pytest.mark.gpu
def test_tokens_outside_and_masked():
    x = _rows(4, 1000, F32, 41)
    x[3, 5] = -math.inf
    tok = torch.tensor([-1, 1000, 2**31 - 1, 5], dtype=torch.int32, device="cuda")
    stats = B.token_logprobs(x, tok)[0].cpu()
    assert torch.isnan(stats[:3, 0]).all() and stats[3, 0] == -math.inf and torch.isfinite(stats[:, 1:]).all()


@pytest.mark.gpu
def test_same_bits_again_and_on_another_stream():
    x, tok = _rows(5, 32003, BF16, 51), _tokens(5, 32003, 52)
    first = B.token_logprobs(x, tok, top_k=20)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    again = [B.token_logprobs(x, tok, top_k=20, stream=st) for _ in range(8)]
    st.synchronize()
    for got in again:
        for a, b in zip(first, got):
            assert torch.equal(a.view(torch.int32), b.view(torch.int32))


@pytest.mark.gpu
def test_graph_replays():
    x, tok = _rows(3, 32003, BF16, 61), _tokens(3, 32003, 62)
    out = tuple(t.clone() for t in B.token_logprobs(x, tok, top_k=20))
    ws = torch.empty(B.token_logprobs_workspace_size(3, 32003, 20), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.token_logprobs(x, tok, top_k=20, out=out, workspace=ws)
    for seed in (63, 64, 65):
        x.copy_(_rows(3, 32003, BF16, seed))
        want = B.token_logprobs(x, tok, top_k=20)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, out):
            assert torch.equal(a.view(torch.int32), b.view(torch.int32))


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """Rows that start more than 2^31 entries apart."""
    V, stride = 4099, (1 << 31) + 8
    buf = torch.empty(stride + V, dtype=BF16, device="cuda")
    x = buf.as_strided((2, V), (stride, 1))
    src = _rows(2, V, BF16, 71)
    x.copy_(src)
    tok = _tokens(2, V, 72)
    _check(src, tok, 5, 1.0, B.token_logprobs(x, tok, top_k=5))


@pytest.mark.gpu
def test_empty_batch():
    stats, ids, lps = B.token_logprobs(torch.empty((0, 100), device="cuda"), top_k=3)
    assert stats.shape == (0, 3) and ids.shape == (0, 3) and lps.shape == (0, 3)


@pytest.mark.gpu
def test_binding_refuses():
    x = torch.zeros((4, 64), device="cuda")
    tok = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (x.double(), x.half()):
        with pytest.raises(TypeError):
            B.token_logprobs(bad)
    with pytest.raises(TypeError):
        B.token_logprobs(x, tok.long())
    for args, kw in (((x[0],), {}), ((x.t(),), {}), ((x[:1].expand(4, 64),), {}), ((x, tok[:3]), {}),
                     ((x, tok.cpu()), {}), ((x.cpu(),), {}), ((x, tok[::2].repeat(2)[::2]), {}),
                     ((x,), dict(out=(torch.zeros((4, 2), device="cuda"),) * 3))):
        with pytest.raises(ValueError):
            B.token_logprobs(*args, **kw)
    for kw in (dict(top_k=257), dict(top_k=-1)):
        with pytest.raises((B.DlsError, RuntimeError)):
            B.token_logprobs(x, **kw)
    for T in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(B.DlsError):
            B.token_logprobs(x, temperature=T)
    with pytest.raises(B.DlsError):
        B.token_logprobs(torch.zeros((2, 151936), device="cuda"), top_k=5, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


# ------------------------------------------------------------------------------------------------
# host side (no GPU): refusals of the C entry point before any device call
# ------------------------------------------------------------------------------------------------
PTR = 0x7f0000000000


def _call(logits=PTR, dtype=1, rows=4, V=1000, stride=1000, tokens=PTR, T=1.0, k=5, stats=PTR, ids=PTR, lps=PTR, ws=PTR, wsb=1 << 30):
    return B.lib().dls_token_logprobs(logits, dtype, rows, V, stride, tokens, T, k, stats, ids, lps, ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), 3), (dict(dtype=-1), 3), (dict(rows=-1), 2), (dict(rows=(1 << 20) + 1), 2), (dict(V=0), 2),
    (dict(V=(1 << 24) + 1, stride=1 << 25), 2), (dict(stride=999), 2), (dict(k=-1), 2), (dict(k=257), 2), (dict(T=0.0), 1), (dict(T=-2.0), 1),
    (dict(T=math.nan), 1), (dict(T=math.inf), 1), (dict(logits=None), 1), (dict(stats=None), 1), (dict(ids=None), 1),
    (dict(lps=None), 1), (dict(logits=PTR + 1), 1), (dict(tokens=PTR + 2), 1), (dict(stats=PTR + 2), 1),
    (dict(ws=None, V=151936, stride=151936), 1), (dict(ws=PTR + 8, V=151936, stride=151936), 1), (dict(wsb=0, V=151936, stride=151936), 4),
])
def test_entry_point_refuses(kw, status):
    assert _call(**kw) == status
    assert B.lib().dls_last_error()


def test_entry_point_takes_no_rows_and_sizes():
    assert _call(rows=0, logits=None, stats=None) == 0
    assert B.token_logprobs_workspace_size(0, 1000, 5) == 0 and B.token_logprobs_workspace_size(4, 1000, 999) == 0
    assert B.token_logprobs_workspace_size(1, 151936, 5) > 0
    # rows past the split hold no parts, where one workgroup can hold the block maxima of a row of either type
    assert B.token_logprobs_workspace_size(1024, 100003, 5) == 0
    assert B.token_logprobs_workspace_size(1024, 151936, 5) > 0
