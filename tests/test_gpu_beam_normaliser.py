"""The normaliser of beam_select: rows of logits of any size, rows that one token dominates.

logp = (x - M) - log S, S the sum of exp(x - M) over the row, M its largest logit. Each term of S is off by at most
2^-22 of itself (ex2.approx, 2.4e-7), by 1.3e-8 a nat below M (the constant log2(e)), and by half a step of its
argument in log2 units: 1.7e-7 up to 8 of them, 3.3e-7 up to 16, 6.6e-7 up to 32. The terms at t nats count
e^-t each, V of them at most V e^-t / (1 + V e^-t) of S: with V = 60,000 the worst lies at t = 6 to 9, 6.5e-7 of S
(near t = 11.1, where the argument passes 16, 5.0e-7; with V = 151,936 there 7.3e-7). The sums in fp32 (chains of
16 or fewer, then halves) add 1.7e-7: below 2^-20 = 9.5e-7 in all. S is not below 1."""
import math

import numpy as np
import pytest
import torch

import workloads
from test_gpu_beam import NINF, _ll, _plain, _run_select

pytestmark = pytest.mark.gpu

TOL = 2.0 ** -20


def _want(x, scores, n, done=None, end_id=-1):
    """As the definition, each row taken from its largest logit: differences in 64 bits lose nothing that
    counts, whatever the logits' size."""
    R, W, V = x.shape
    K = min(n, V)
    ids, total = np.zeros((R, W, K), np.int64), np.full((R, W, K), NINF)
    for r in range(R):
        for w in range(W):
            if not scores[r, w] > NINF or (done is not None and done[r, w]):
                continue
            row = x[r, w].astype(np.float64)
            ids[r, w] = np.lexsort((np.arange(V), -row))[:K]
            row = row - row.max()
            total[r, w] = np.float64(scores[r, w]) + (row[ids[r, w]] - math.log1p(np.sort(np.exp(row))[:-1].sum()))
    total[total < -float(np.finfo(np.float32).max)] = NINF         # no total that fp32 holds
    return _plain(ids, total, scores, n, done, end_id)


def _check(got, want):
    """Picks, and totals to the stated bound."""
    tok, par, sc, over = (t.cpu().numpy() for t in got)
    assert np.array_equal(tok, want[0]) and np.array_equal(par, want[1]) and np.array_equal(over, want[3])
    fin = np.isfinite(want[2])
    assert np.array_equal(np.isfinite(sc), fin)
    err = np.abs(sc[fin] - want[2][fin]) - (TOL + 2.0 ** -24 * np.abs(want[2][fin]))
    assert np.all(err <= 0), err.max()


LOW = {"f32": float(np.finfo(np.float32).min), "bf16": float(torch.finfo(torch.bfloat16).min)}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["lowest", "lowest_but_few", "highest", "highest_and_lowest", "1e9", "-1e9", "1e6",
                                  "-3e4", "mixed"])
@pytest.mark.parametrize("V", [37, 5001, 40000])
def test_rows_of_finite_logits_of_any_size(kind, V, dtype):
    """Masks of the type's lowest value over all of a row or most of it, logits near both ends of fp32's range, and
    rows far from 0, next to an ordinary beam."""
    ll = _ll()
    rng = np.random.default_rng(V)
    R, W, n = 3, 3, 4
    x = np.round(rng.standard_normal((R, W, V)) * 64) / 64
    x[:, :, V // 3] += 9.0                                     # ahead of its row
    few = rng.permutation(V)[:5]
    y = x[:, 1].copy()
    low = LOW[dtype]
    if kind == "lowest":
        y[:] = low
    elif kind == "lowest_but_few":
        y[:] = low
        y[:, few] = x[:, 1][:, few]
    elif kind == "highest":
        y[:, few[:3]] = [-low, -low, -low / 2]
    elif kind == "highest_and_lowest":
        y[:] = low
        y[:, few[:2]] = -low
    elif kind == "mixed":
        y[:] = np.where(rng.uniform(size=y.shape) < 0.5, low, -1e9)
        y[:, few] = [30.0, 29.0, 28.5, 2e4, 2e4]
    else:
        y += float(kind)
    x[:, 1] = y
    x = x.astype(np.float32)
    if dtype == "bf16":
        x = workloads.round_to_bf16(x)
    assert np.isfinite(x).all()
    scores = np.array([[-1.0, -0.5, -1.25]] * R, np.float32)
    want = _want(x, scores, n)
    t = want[2]                                                # (totals of two beams are apart, or the test says nothing)
    assert all(want[1][r, j] == want[1][r, j + 1] or t[r, j] - t[r, j + 1] > 4 * TOL
               for r in range(R) for j in range(n - 1))
    ws = ll.Workspace(ll.beam_select_workspace_bytes(R, W, V, n))
    _check(_run_select(ll, x, scores, n, dtype, ws=ws), want)
    assert ws.status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2, 1000, 1003, 60000])
def test_a_row_that_one_token_dominates(V, dtype):
    """No total lies above its score, and each is the definition's to the stated bound."""
    ll = _ll()
    rng = np.random.default_rng(V)
    R, W = 8, 60
    x = rng.standard_normal((R, W, V)).astype(np.float32)
    peak = np.linspace(3.0, 90.0, R * W).reshape(R, W) + rng.uniform(0, 0.2, (R, W))
    at = rng.integers(0, V, (R, W))
    for r in range(R):
        for w in range(W):
            x[r, w, at[r, w]] = peak[r, w]
    if dtype == "bf16":
        x = workloads.round_to_bf16(x)
    scores = np.zeros((R, W), np.float32)
    # a request a row, so that each one's own best is seen
    flat = x.reshape(R * W, 1, V)
    got = _run_select(ll, flat, scores.reshape(R * W, 1), 1, dtype)
    tok, _, sc, _ = (t.cpu().numpy() for t in got)
    assert np.all(sc <= 0.0), sc.max()
    row = flat[:, 0].astype(np.float64)
    m = row.max(1)
    rest = np.exp(row - m[:, None])
    exact = -np.log1p(np.sort(rest, axis=1)[:, :-1].sum(1))
    assert np.array_equal(tok[:, 0], row.argmax(1))
    assert np.all(np.abs(sc[:, 0] - exact) <= TOL + 2.0 ** -24 * np.abs(exact))
    # and against scores of a few nats: never above them
    sc7 = -rng.uniform(0, 7, (R * W, 1)).astype(np.float32)
    out = _run_select(ll, flat, sc7, 1, dtype)[2].cpu().numpy()
    assert np.all(out <= sc7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [4096, 4097, 3 * 4096 + 5])
def test_unlike_beams_keep_their_totals_apart(V, dtype):
    """Rows of zeros, each with one logit a little lower, by 2^-10 more in every beam: log S falls by 2^-10 / V a
    beam, 2.4e-7 at most, which fp32's totals do not show. Terms of 1 are exact; with the one other, halves of
    half steps of sums of up to 2,048, below 2^-13 in all, are 1/8 of a gap. The likeliest beam's zeros come first."""
    ll = _ll()
    W, n = 8, 24
    x = np.zeros((2, W, V), np.float32)
    order = [list(range(W)), [3, 6, 1, 7, 0, 5, 2, 4]]         # how much lower each beam's logit is
    for r in range(2):
        for w in range(W):
            x[r, w, 17 * w + 3] = -(2.0 ** -10) * order[r][w]
    assert np.array_equal(workloads.round_to_bf16(x), x)
    scores = np.full((2, W), -2.0, np.float32)
    want = _want(x, scores, n)
    assert want[1].tolist() == [[W - 1] * n, [3] * n]
    _check(_run_select(ll, x, scores, n, dtype), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,W,V", [(3, 16, 2049), (2, 9, 40001), (5, 8, 8192), (1, 64, 1003)])
@pytest.mark.parametrize("kind", ["level", "far"])
def test_beams_of_one_content_tie_with_banned_tokens(kind, R, W, V, dtype):
    """The same logits at every alignment, of one value behind a peak (all roundings alike) or of many, some
    banned, some beams absent: the lower beam goes first throughout."""
    ll = _ll()
    rng = np.random.default_rng(V)
    row = np.full((R, 1, V), -9.7) if kind == "level" else rng.standard_normal((R, 1, V)) * 3 - 1e4
    row[:, 0, V // 3] = row.max() + 10.4
    row[:, 0, V // 2:V // 2 + V // 8] = NINF
    x = np.repeat(row.astype(np.float32), W, axis=1)
    if dtype == "bf16":
        x = workloads.round_to_bf16(x)
    scores = np.full((R, W), -0.75, np.float32)
    scores[:, 1] = NINF
    n = min(32, W - 1)
    tok, par, sc, _ = (t.cpu().numpy() for t in _run_select(ll, x, scores, n, dtype))
    for r in range(R):
        ids = np.argsort(-x[r, 0], kind="stable")[:n]              # (bf16 near -1e4: most logits are equal)
        first = sorted((-x[r, w, v], w, v) for w in range(W) if w != 1 for v in ids)[:n]
        assert par[r].tolist() == [c[1] for c in first] and tok[r].tolist() == [c[2] for c in first]
        assert all(sc[r, j] == sc[r, j - 1] for j in range(1, n) if first[j][0] == first[j - 1][0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 1003, 4097, 4096, 12345])
def test_zeros_of_either_sign_are_the_same_logit(V, dtype):
    """Beams alike but for the signs of their zeros tie, at every alignment."""
    ll = _ll()
    rng = np.random.default_rng(V)
    R, W, n = 3, 9, 12
    row = np.round(rng.standard_normal((R, 1, V)) * 2) / 4
    row[:, :, V // 2] = 3.0
    x = np.repeat(row, W, axis=1)
    x = np.where((x == 0) & (rng.uniform(size=x.shape) < 0.5), -0.0, x + 0.0).astype(np.float32)
    assert np.signbit(x[x == 0]).any() and not np.signbit(x[x == 0]).all()
    scores = np.zeros((R, W), np.float32)
    want = _want(x, scores, n)
    _check(_run_select(ll, x, scores, n, dtype), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [(1 << 31) - 1, (1 << 31) - 8])
def test_a_vocabulary_that_ends_at_31_bits(V, dtype):
    """Ids up to the largest int32: the row's last piece ends there, inside a vector or at one's end."""
    ll = _ll()
    x = torch.full((1, 1, V), -1.0, dtype=dtype, device="cuda")
    at = {V - 1: 30.0, 0: 29.0, V - 2050: 28.0, 1500000001: 27.0, V - 2: 26.5}
    for v, y in at.items():
        x[0, 0, v] = y
    ws = ll.Workspace(ll.beam_select_workspace_bytes(1, 1, V, 5))
    tok, par, sc, _ = ll.beam_select(x, torch.zeros((1, 1), device="cuda"), 5, ws=ws)
    lse = math.log(sum(math.exp(y) for y in at.values()) + (V - 5) * math.exp(-1.0))
    assert tok.cpu().tolist() == [list(at)] and par.cpu().tolist() == [[0] * 5] and ws.status() == 0
    for got, y in zip(sc.cpu().tolist()[0], at.values()):
        assert abs(got - (y - lse)) <= TOL + 2.0 ** -24 * abs(y - lse)
    del x


@pytest.mark.parametrize("V", [151936, 128257])
def test_a_level_background_behind_a_peak(V):
    """All terms but one round alike, the case the bound on log S is made of: 96 distances of the peak."""
    ll = _ll()
    t = np.float32(2.0) + np.arange(96, dtype=np.float32) * np.float32(0.15625)          # up to 16.8 nats
    x = torch.zeros((96, 1, V), device="cuda")
    x[:, 0, V // 2] = torch.from_numpy(t).cuda()
    tok, _, sc, _ = ll.beam_select(x, torch.zeros((96, 1), device="cuda"), 2)
    exact = -np.log1p((V - 1) * np.exp(-t.astype(np.float64)))
    assert tok.cpu().tolist() == [[V // 2, 0]] * 96
    err = np.abs(sc.cpu().numpy()[:, 0] - exact)
    assert np.all(err <= TOL + 2.0 ** -24 * np.abs(exact)), err.max()
