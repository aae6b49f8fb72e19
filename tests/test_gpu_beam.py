"""Beam selection and the move of the beams' states against plain 64-bit and copying forms.

Totals are compared exactly where their inputs make them exact (``beam_merge``: sums of two fp32
numbers in 64 bits, rounded once to fp32, half a step 2^-24 relative). From logits the normaliser is
a sum of V terms, each off by at most 2^-21 of itself (the exponential's argument is rounded to
2^-24 of at most 8 in front of a term that matters, ex2.approx is good to 2^-22), so the total is off
by at most 2^-21 before its rounding to fp32. Where neighbouring totals of different beams are
closer than twice that, either order is right: then the j-th pick's total in 64 bits has to be the
j-th largest within that distance, and each beam's picks a leading run of its own order."""
import math

import numpy as np
import pytest
import torch

import workloads

pytestmark = pytest.mark.gpu

NINF = -math.inf
LSE_TOL = 2.0 ** -21


def _ll():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_20530_gb300 as ll
    return ll


def _plain(ids, total, scores, n, done, end_id):
    """The definition on [R][W] lists of (token, 64-bit total) in the candidates' order."""
    R, W = scores.shape
    tok, par = np.full((R, n), -1, np.int32), np.full((R, n), -1, np.int32)
    out, over = np.full((R, n), NINF, np.float64), np.zeros((R, n), bool)
    for r in range(R):
        cand = []
        for w in range(W):
            if done is not None and done[r, w]:
                cand.append((np.float64(scores[r, w]), w, 0, end_id, True))
            elif scores[r, w] > NINF:
                cand += [(total[r, w, k], w, k, ids[r, w, k], ids[r, w, k] == end_id >= 0)
                         for k in range(ids.shape[2])]
        cand = sorted((c for c in cand if c[0] > NINF), key=lambda c: (-c[0], c[1], c[2]))[:n]
        for j, c in enumerate(cand):
            out[r, j], par[r, j], tok[r, j], over[r, j] = c[0], c[1], c[3], c[4]
    return tok, par, out, over


def _check(got, want, tol=0.0):
    tok, par, sc, over = (t.cpu().numpy() for t in got)
    assert np.array_equal(tok, want[0]) and np.array_equal(par, want[1])
    assert np.array_equal(over, want[3])
    fin = np.isfinite(want[2])
    assert np.array_equal(np.isfinite(sc), fin) and np.all(sc[~fin] == NINF)
    err = np.abs(sc[fin] - want[2][fin])
    assert np.all(err <= tol + 2.0 ** -24 * np.abs(want[2][fin])), err.max()


def _select_inputs(R, W, V, dtype, seed, done=False, banned=0, absent=False):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, W, V)).astype(np.float32) * 2
    for r in range(R):
        for w in range(W):
            x[r, w, rng.integers(0, V, 5)] += rng.uniform(0, 8, 5).astype(np.float32)
    if banned:
        x[:, :, rng.permutation(V)[:banned]] = NINF
    if dtype == "bf16":
        x = workloads.round_to_bf16(x)
    scores = (-np.cumsum(rng.uniform(0, 1, (R, W)), axis=1)).astype(np.float32)
    if absent:
        scores[:, W - 1] = NINF
    dn = (rng.uniform(size=(R, W)) < 0.4) if done else None
    if dn is not None:
        x[dn] = np.nan                                # a finished beam's logits are not read
    if absent:
        x[:, W - 1] = np.nan
    return x, scores, dn


def _want_select(x, scores, n, done, end_id):
    """The n best of each row by (logit, lower id), their totals in 64 bits; and the smallest gap
    between totals of different beams that the answer's order rests on."""
    R, W, V = x.shape
    K = min(n, V)
    ids, total = np.zeros((R, W, K), np.int64), np.full((R, W, K), NINF)
    for r in range(R):
        for w in range(W):
            if not scores[r, w] > NINF or (done is not None and done[r, w]):
                continue
            row = x[r, w].astype(np.float64) + 0.0
            ids[r, w] = np.lexsort((np.arange(V), -row))[:K]
            m = row.max()
            total[r, w] = np.float64(scores[r, w]) + (row[ids[r, w]] - (m + math.log(np.exp(row - m).sum())))
    want = _plain(ids, total, scores, n, done, end_id)
    more = _plain(ids, total, scores, n + 1, done, end_id)
    # requests whose order rests on no gap between beams below 2 LSE_TOL
    clear = []
    for r in range(R):
        t, p = more[2][r], more[1][r]
        clear.append(all(p[j] == p[j + 1] or not np.isfinite(t[j + 1]) or t[j] - t[j + 1] > 2 * LSE_TOL
                         for j in range(n)))
    return want + (np.array(clear), ids, total)


def _check_select(got, want, scores, done, end_id):
    tok, par, sc, over = (t.cpu().numpy() for t in got)
    wt, wp, ws_, wo, clear, ids, total = want
    c = clear
    assert np.array_equal(tok[c], wt[c]) and np.array_equal(par[c], wp[c])
    assert np.array_equal(over[c], wo[c])
    there = ws_ > NINF
    assert np.array_equal(sc > NINF, there) and np.all(tok[~there] == -1) and np.all(par[~there] == -1)
    for r in range(len(tok)):
        taken = {}
        for j in np.nonzero(there[r])[0]:
            w = int(par[r, j])
            k = taken.get(w, 0)
            taken[w] = k + 1
            if done is not None and done[r, w]:
                exact, token = np.float64(scores[r, w]), end_id
                assert k == 0 and over[r, j]
            else:
                exact, token = total[r, w, k], ids[r, w, k]
                assert over[r, j] == (token == end_id >= 0)
            assert tok[r, j] == token
            assert abs(exact - ws_[r, j]) <= 2 * LSE_TOL
            assert abs(sc[r, j] - exact) <= LSE_TOL + 2.0 ** -24 * abs(exact)


def _run_select(ll, x, scores, n, dtype, done=None, end_id=-1, ws=None):
    t = torch.from_numpy(x).cuda()
    if dtype == "bf16":
        t = t.to(torch.bfloat16)
    return ll.beam_select(t, torch.from_numpy(scores).cuda(), n,
                          done=None if done is None else torch.from_numpy(done).cuda(),
                          end_id=end_id, ws=ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,W,V,n", [(1, 1, 1, 1), (1, 2, 3, 5), (1, 4, 151936, 8), (2, 5, 1001, 5),
                                     (3, 3, 9, 27), (7, 8, 4099, 16), (2, 64, 333, 32),
                                     (40, 16, 2000, 32), (300, 2, 517, 4), (700, 4, 64, 8)])
def test_beam_select_shapes(dtype, R, W, V, n):
    ll = _ll()
    x, scores, _ = _select_inputs(R, W, V, dtype, 7 * R + W + V + n)
    want = _want_select(x, scores, n, None, -1)
    ws = ll.Workspace(ll.beam_select_workspace_bytes(R, W, V, n))
    first = _run_select(ll, x, scores, n, dtype, ws=ws)
    _check_select(first, want, scores, None, -1)
    again = _run_select(ll, x, scores, n, dtype, ws=ws)                    # the workspace again
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    assert ws.status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,W,V,n,banned", [(5, 4, 3001, 8, 100), (3, 6, 40, 12, 37), (2, 3, 50, 32, 49)])
def test_beam_select_done_absent_and_banned(dtype, R, W, V, n, banned):
    """Finished and absent beams' logits are NaN and are not read; with nearly every token banned
    there are fewer candidates than n."""
    ll = _ll()
    x, scores, done = _select_inputs(R, W, V, dtype, 31 * V + n, done=True, banned=banned, absent=True)
    done[0, :] = True                                 # a request whose beams have all ended
    x[0] = np.nan
    want = _want_select(x, scores, n, done, 7)
    ws = ll.Workspace(ll.beam_select_workspace_bytes(R, W, V, n))
    _check_select(_run_select(ll, x, scores, n, dtype, done, 7, ws), want, scores, done, 7)
    assert ws.status() == 0


def test_beam_select_one_workspace_for_calls_of_many_shapes():
    """Calls of different shapes, sharing one workspace in turn, each find it usable."""
    ll = _ll()
    shapes = [(1, 4, 151936, 8, "bf16"), (40, 3, 900, 5, "f32"), (6, 8, 40001, 16, "f32"),
              (2, 2, 5000, 4, "bf16"), (300, 2, 64, 4, "bf16")]
    ws = ll.Workspace(max(ll.beam_select_workspace_bytes(*s[:4]) for s in shapes))
    for turn in range(2):
        for i, (R, W, V, n, dtype) in enumerate(shapes):
            x, scores, _ = _select_inputs(R, W, V, dtype, 100 * turn + i)
            want = _want_select(x, scores, n, None, -1)
            _check_select(_run_select(ll, x, scores, n, dtype, ws=ws), want, scores, None, -1)
    assert ws.status() == 0


def test_beam_select_no_beam_at_all():
    ll = _ll()
    x = np.full((2, 3, 100), np.nan, np.float32)
    scores = np.full((2, 3), NINF, np.float32)
    tok, par, sc, over = (t.cpu().numpy() for t in _run_select(ll, x, scores, 4, "f32"))
    assert np.all(tok == -1) and np.all(par == -1) and np.all(sc == NINF) and not over.any()


def test_beam_select_equal_logits_and_equal_beams():
    """Constant rows: ids in order; beams alike in everything tie, and the lower one goes first."""
    ll = _ll()
    x = np.zeros((1, 3, 4096), np.float32)
    x[0, :, 100] = -0.0
    scores = np.array([[-1.0, -1.0, -2.0]], np.float32)
    tok, par, sc, _ = (t.cpu().numpy() for t in _run_select(ll, x, scores, 8, "f32"))
    assert tok[0].tolist() == list(range(8)) and par[0].tolist() == [0] * 8
    x[0, :, 5] = 3.0
    tok, par, sc, _ = (t.cpu().numpy() for t in _run_select(ll, x, scores, 4, "f32"))
    assert tok[0].tolist() == [5, 5, 5, 0] and par[0].tolist() == [0, 1, 2, 0]
    assert sc[0, 0] == sc[0, 1]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["constant", "falling", "rising", "grid", "head_and_tail"])
@pytest.mark.parametrize("W,V,n", [(8, 40001, 32), (3, 5003, 8), (12, 151936, 24)])
def test_beam_select_rows_of_equal_and_of_ordered_logits(dtype, kind, W, V, n):
    """Ties over the whole vocabulary, and rows whose best logits all lie next to one another."""
    ll = _ll()
    rng = np.random.default_rng(V + n)
    at = np.arange(V)
    if kind == "constant":
        x = np.full((2, W, V), 1.5)
    elif kind == "falling":
        x = np.tile(-0.25 * (at // 3), (2, W, 1))
    elif kind == "rising":
        x = np.tile(0.25 * ((at - V) // 5), (2, W, 1))
    elif kind == "grid":
        x = np.round(rng.standard_normal((2, W, V)) * 4) / 4
    else:
        x = rng.standard_normal((2, W, V))
        x[:, :, [0, 1, 2, V - 3, V - 2, V - 1]] += 20.0
    x = x.astype(np.float32)
    if dtype == "bf16":
        x = workloads.round_to_bf16(x)
    scores = -np.arange(2 * W, dtype=np.float32).reshape(2, W) / 1000
    want = _want_select(x, scores, n, None, -1)
    _check_select(_run_select(ll, x, scores, n, dtype), want, scores, None, -1)


def test_beam_select_equal_beams_with_equal_rows():
    """Eight beams alike in everything, constant rows: position alone orders all candidates."""
    ll = _ll()
    x = torch.zeros((1, 8, 151936), dtype=torch.bfloat16, device="cuda")
    tok, par, sc, _ = ll.beam_select(x, torch.zeros((1, 8), device="cuda"), 32)
    assert tok.cpu().tolist() == [list(range(32))] and par.cpu().tolist() == [[0] * 32]
    x[0, :, 1000:1100] = 2.0
    tok, par, sc, _ = ll.beam_select(x, torch.zeros((1, 8), device="cuda"), 32)
    assert tok.cpu().tolist() == [list(range(1000, 1032))] and par.cpu().tolist() == [[0] * 32]


@pytest.mark.parametrize("bad", [np.nan, np.inf, "row", "score_nan", "score_inf"])
@pytest.mark.parametrize("V", [37, 20000])
def test_beam_select_nonfinite(bad, V):
    """The beam is left out and the status set; the other beams are picked from as ever."""
    ll = _ll()
    x, scores, _ = _select_inputs(2, 3, V, "f32", 5)
    sc = scores.copy()
    sc[0, 1] = NINF
    want = _want_select(x, sc, 3, None, -1)
    if bad == "row":
        x[0, 1] = NINF
    elif bad == "score_nan":
        scores[0, 1] = np.nan
    elif bad == "score_inf":
        scores[0, 1] = np.inf
    else:
        x[0, 1, V // 2] = bad
    ws = ll.Workspace(ll.beam_select_workspace_bytes(2, 3, V, 3))
    _check_select(_run_select(ll, x, scores, 3, "f32", ws=ws), want, sc, None, -1)
    assert ws.status() == ll.ERR_NONFINITE
    assert ws.status() == 0


def test_beam_select_row_of_nan_only():
    ll = _ll()
    x = np.full((1, 1, 5000), np.nan, np.float32)
    ws = ll.Workspace(ll.beam_select_workspace_bytes(1, 1, 5000, 2))
    tok, _, _, _ = _run_select(ll, x, np.zeros((1, 1), np.float32), 2, "f32", ws=ws)
    assert tok.cpu().tolist() == [[-1, -1]] and ws.status() == ll.ERR_NONFINITE


@pytest.mark.parametrize("R,W,K,n", [(1, 1, 1, 1), (1, 4, 8, 8), (3, 2, 2, 4), (17, 16, 32, 32),
                                     (5, 64, 32, 32), (9, 24, 7, 13), (200, 3, 5, 2)])
@pytest.mark.parametrize("done", [False, True])
def test_beam_merge(R, W, K, n, done):
    """Totals on a coarse grid: most of them meet, so the order rests on the tie rule."""
    ll = _ll()
    rng = np.random.default_rng(R + 10 * W + 100 * K + n)
    logp = (-rng.integers(0, 24, (R, W, K)) / 8).astype(np.float32)
    logp[rng.uniform(size=logp.shape) < 0.1] = NINF
    ids = rng.integers(0, 40, (R, W, K)).astype(np.int32)
    scores = (-rng.integers(0, 8, (R, W)) / 8).astype(np.float32)
    scores[rng.uniform(size=scores.shape) < 0.1] = NINF
    dn = rng.uniform(size=(R, W)) < 0.3 if done else None
    if done:
        logp[dn] = np.nan
    end = 3 if done or W % 2 else -1
    total = scores.astype(np.float64)[:, :, None] + logp.astype(np.float64)
    want = _plain(ids, total, scores, n, dn, end)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = ll.beam_merge(torch.from_numpy(ids).cuda(), torch.from_numpy(logp).cuda(),
                        torch.from_numpy(scores).cuda(), n,
                        done=None if dn is None else torch.from_numpy(dn).cuda(), end_id=end,
                        status=st)
    _check(got, want)
    assert int(st) == 0


def test_beam_merge_all_totals_equal():
    ll = _ll()
    ids = torch.arange(64 * 32, dtype=torch.int32, device="cuda").view(1, 64, 32)
    tok, par, sc, _ = ll.beam_merge(ids, torch.zeros_like(ids, dtype=torch.float32),
                                    torch.zeros((1, 64), device="cuda"), 32)
    assert tok.cpu().tolist() == [list(range(32))] and par.cpu().tolist() == [[0] * 32]


def test_beam_merge_told_apart_below_fp32():
    """Totals that agree in fp32 and differ in 64 bits keep their order."""
    ll = _ll()
    scores = torch.tensor([[-100.0, -100.0, -100.0]], device="cuda")
    logp = torch.tensor([[[-3e-7], [-1e-7], [-2e-7]]], device="cuda")
    ids = torch.tensor([[[5], [6], [7]]], dtype=torch.int32, device="cuda")
    tok, par, sc, _ = ll.beam_merge(ids, logp, scores, 3)
    assert tok.cpu().tolist() == [[6, 7, 5]] and sc.cpu().tolist() == [[-100.0] * 3]


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_beam_merge_nonfinite(bad):
    ll = _ll()
    logp = torch.tensor([[[-1.0, bad], [-2.0, -3.0]]], device="cuda")
    ids = torch.tensor([[[1, 2], [3, 4]]], dtype=torch.int32, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    tok, par, sc, _ = ll.beam_merge(ids, logp, torch.zeros((1, 2), device="cuda"), 3, status=st)
    assert tok.cpu().tolist() == [[1, 3, 4]] and int(st) == ll.ERR_NONFINITE


def test_beam_merge_of_topk_lists_is_beam_select():
    """topk_lse's lists merged are the step from logits (the lists' log-probabilities are rounded to
    fp32, so the inputs' gaps are looked at against that rounding)."""
    ll = _ll()
    x, scores, _ = _select_inputs(3, 4, 5000, "bf16", 77)
    want = _want_select(x, scores, 8, None, -1)
    assert want[4].all() and np.diff(want[2]).max() < -2.0 ** -18
    t = torch.from_numpy(x).cuda().to(torch.bfloat16)
    ids, logp, _ = ll.topk_lse(t, 8)
    _check(ll.beam_merge(ids, logp, torch.from_numpy(scores).cuda(), 8), want[:4], 2.0 ** -19)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,W,V,n", [(1, 8, 151935, 12), (30, 5, 4771, 12), (90, 16, 2049, 32), (7, 64, 1001, 20),
                                     (200, 3, 40, 7)])
def test_beam_select_beams_of_one_content(R, W, V, n, dtype):
    """Beams with the same logits and the same score, at every alignment: equal totals go to the lower
    beam, whatever the order in which the rows were summed."""
    ll = _ll()
    x, _, _ = _select_inputs(R, 1, V, dtype, V + W)
    x[:, 0, :] = np.round(x[:, 0, :] * 8) / 8                    # (equal logits too)
    x[:, 0, V // 2] = 30.0                                       # two that are ahead of all others
    x[:, 0, V // 3] = 29.5
    ids = np.argsort(-x[:, 0], axis=1, kind="stable")
    x = np.repeat(x, W, axis=1)
    scores = np.zeros((R, W), np.float32)
    tok, par, sc, _ = (t.cpu().numpy() for t in _run_select(ll, x, scores, n, dtype))
    for r in range(R):
        first = sorted((-x[r, w, v], w, v) for w in range(W) for v in ids[r, :n])[:n]
        assert par[r].tolist() == [c[1] for c in first]
        assert tok[r].tolist() == [c[2] for c in first]
        assert all(sc[r, j] == sc[r, j - 1] for j in range(1, n) if first[j][0] == first[j - 1][0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,ban", [(6148, None), (8198, None), (4102, (0, 2100)), (9000, (2000, 7000)),
                                   (8192, (4096, 8192)), (5001, (0, 4990))])
def test_beam_select_runs_of_banned_tokens(V, ban, dtype):
    """Whole pieces of a row without a finite logit (a run of banned tokens, or none left of the row), where
    a warp walks several pieces: they add nothing to the row's sum, and the row stays."""
    ll = _ll()
    R, W, n = 80, 8, 6
    x, scores, _ = _select_inputs(R, W, V, dtype, V)
    if ban:
        x[:, :, ban[0]:ban[1]] = NINF
    ws = ll.Workspace(ll.beam_select_workspace_bytes(R, W, V, n))
    got = _run_select(ll, x, scores, n, dtype, ws=ws)
    _check_select(got, _want_select(x, scores, n, None, -1), scores, None, -1)
    assert ws.status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,W,V,n", [(3, 16, 1697, 32), (5, 4, 900, 32), (2, 2, 40, 31), (4, 13, 2375, 26),
                                     (1, 1, 2048, 32)])
def test_beam_select_few_pieces(R, W, V, n, dtype):
    """Fewer pieces of the rows than continuations, or not many more: most of a piece reaches the bound.
    Logits of few values too, so that ids decide."""
    ll = _ll()
    for grid in (None, 4, 1, -1):
        x, scores, _ = _select_inputs(R, W, V, dtype, R + V)
        if grid is not None:                                    # -1: all equal, negative
            x = np.full_like(x, -3.0) if grid < 0 else (np.round(x * grid / 4) / grid).astype(np.float32) + 0.0
        want = _want_select(x, scores, n, None, -1)
        _check_select(_run_select(ll, x, scores, n, dtype), want, scores, None, -1)


def test_beam_python_refusals():
    ll = _ll()
    x, sc = torch.zeros((2, 3, 50), device="cuda"), torch.zeros((2, 3), device="cuda")
    for call in (lambda: ll.beam_select(x[0], sc, 4), lambda: ll.beam_select(x.cpu(), sc, 4),
                 lambda: ll.beam_select(x.transpose(0, 1), sc, 4), lambda: ll.beam_select(x, sc.double(), 4),
                 lambda: ll.beam_select(x, sc[:, :2], 4), lambda: ll.beam_select(x.half(), sc, 4),
                 lambda: ll.beam_select(x, sc, 4, done=sc, end_id=1),
                 lambda: ll.beam_merge(x.int(), x[:, :, :4], sc, 4),
                 lambda: ll.beam_reorder(torch.zeros((2, 4, 5), device="cuda"),
                                         torch.zeros((2, 3), dtype=torch.int32, device="cuda")),
                 lambda: ll.beam_reorder(torch.zeros((2, 3, 5, 4, 6), device="cuda").transpose(3, 4),
                                         torch.zeros((2, 3), dtype=torch.int32, device="cuda")),
                 lambda: ll.beam_reorder(torch.zeros((2, 3, 5), device="cuda"),
                                         torch.zeros((2, 3), dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ll.beam_select(x, sc, 33), lambda: ll.beam_select(x, sc, 0),
                 lambda: ll.beam_select(x, sc, 4, end_id=50),
                 lambda: ll.beam_merge(x.int(), x, sc, 4),
                 lambda: ll.beam_select(x, sc, 4, ws=ll.Workspace(256))):
        with pytest.raises(ll.LilicorrError):
            call()


# ------------------------------------------------------------------------------- states
def _moved(state, parents, lengths):
    out = state.clone()
    R, W = parents.shape
    for r in range(R):
        n = state.shape[2] if lengths is None else min(max(int(lengths[r]), 0), state.shape[2])
        for w in range(W):
            p = int(parents[r, w])
            if 0 <= p < W:
                out[r, w, :n] = state[r, p, :n]
    return out


def _bits(t):
    return t.contiguous().view(torch.uint8)


@pytest.mark.parametrize("R,W,S,tail,dtype", [
    (1, 1, 5, (8,), torch.bfloat16), (1, 4, 64, (8, 128), torch.bfloat16),
    (3, 5, 33, (2, 80), torch.float32), (2, 8, 17, (3, 7), torch.bfloat16),
    (2, 9, 40, (5,), torch.uint8), (2, 16, 21, (4, 64), torch.bfloat16),
    (1, 17, 30, (2, 64), torch.float32), (2, 32, 9, (3, 5), torch.bfloat16),
    (1, 33, 25, (2, 64), torch.bfloat16), (1, 64, 12, (31,), torch.uint8),
    (4, 3, 700, (4, 128), torch.bfloat16), (5, 2, 1, (), torch.int32)])
@pytest.mark.parametrize("use_lengths", [False, True])
def test_beam_reorder(R, W, S, tail, dtype, use_lengths):
    ll = _ll()
    g = torch.Generator().manual_seed(R * 100 + W)
    raw = [torch.randint(0, 255, (R, W, S) + tail, generator=g) for _ in range(3)]
    states = [(x.float() / 7).to(dtype) if dtype.is_floating_point else x.to(dtype) for x in raw]
    parents = torch.randint(-1, W + 1, (R, W), generator=g).int()       # outside: the beam stays
    lengths = torch.randint(-1, S + 3, (R,), generator=g).int() if use_lengths else None
    dev = [s.cuda() for s in states]
    out = ll.beam_reorder(dev, parents.cuda(), None if lengths is None else lengths.cuda())
    assert out is dev
    for s, d in zip(states, dev):
        assert torch.equal(_bits(d.cpu()), _bits(_moved(s, parents, lengths)))


@pytest.mark.parametrize("perm", [[1, 2, 3, 0], [1, 0, 3, 2], [0, 0, 0, 0], [3, 3, 0, 0], [0, 1, 2, 3]])
def test_beam_reorder_cycles(perm):
    ll = _ll()
    s = torch.arange(4 * 1000 * 32, dtype=torch.int32).view(1, 4, 1000, 32)
    d = s.cuda()
    ll.beam_reorder(d, torch.tensor([perm], dtype=torch.int32, device="cuda"))
    assert torch.equal(d.cpu(), s[:, perm])


@pytest.mark.parametrize("off", [0, 1, 2, 4, 8])
def test_beam_reorder_strides_and_alignment(off):
    """Caches by head, padded rows, and bases off every vector width; the bytes between stay."""
    ll = _ll()
    R, W, H, S, d = 2, 3, 4, 19, 24
    buf = torch.randint(0, 255, (off + R * W * H * (S + 2) * (d + off) + 64,), dtype=torch.uint8)
    want = buf.clone()

    def view(b):
        x = b[off: off + R * W * H * (S + 2) * (d + off)].view(R, W, H, S + 2, d + off)
        return x.transpose(2, 3)[:, :, 1:S + 1, :, :d]
    parents = torch.tensor([[2, 0, 1], [1, 1, 0]], dtype=torch.int32)
    lengths = torch.tensor([S, 7], dtype=torch.int32)
    view(want).copy_(_moved(view(buf), parents, lengths))
    dev = buf.cuda()
    ll.beam_reorder([view(dev)], parents.cuda(), lengths.cuda())
    assert torch.equal(dev.cpu(), want)


def test_beam_reorder_many_arrays_of_two_shapes():
    ll = _ll()
    g = torch.Generator().manual_seed(3)
    states = [torch.randn((2, 4, 6 + i % 2, 16), generator=g) for i in range(150)]
    parents = torch.tensor([[1, 1, 0, 2], [3, 2, 1, 0]], dtype=torch.int32)
    dev = [s.cuda() for s in states]
    ll.beam_reorder(dev, parents.cuda())
    for s, d in zip(states, dev):
        assert torch.equal(d.cpu(), _moved(s, parents, None))


def test_beam_reorder_offsets_past_32_bits():
    ll = _ll()
    step = (1 << 32) + 4096                            # bytes from one request to the next
    big = torch.zeros(2 * step, dtype=torch.uint8, device="cuda")
    s = torch.as_strided(big, (2, 2, 3, 64), (step, step - 2048, 64, 1))
    g = torch.Generator().manual_seed(4)
    vals = torch.randint(0, 255, (2, 2, 3, 64), generator=g, dtype=torch.uint8)
    s[0].copy_(vals[0]); s[1, 0].copy_(vals[1, 0])     # [1, 1] would lie behind the buffer's end
    ll.beam_reorder(torch.as_strided(big, (1, 2, 3, 64), (step, step - 2048, 64, 1)),
                    torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    assert torch.equal(s[0].cpu(), vals[0].flip(0))
    del big


def test_beam_calls_in_a_graph_and_on_another_stream():
    """One decoding step captured and replayed on new inputs, on a stream of its own."""
    ll = _ll()
    R, W, V, n = 2, 4, 3000, 4
    xs = [_select_inputs(R, W, V, "f32", s) for s in (1, 2, 3)]
    t, sc = torch.empty((R, W, V), device="cuda"), torch.empty((R, W), device="cuda")
    cache = torch.empty((R, W, 10, 32), device="cuda")
    ws = ll.Workspace(ll.beam_select_workspace_bytes(R, W, V, n))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = ll.beam_select(t, sc, n, ws=ws)
        ll.beam_reorder(cache, out[1])
    g = torch.Generator().manual_seed(1)
    for x, scores, _ in xs:
        c0 = torch.randn((R, W, 10, 32), generator=g)
        t.copy_(torch.from_numpy(x)); sc.copy_(torch.from_numpy(scores)); cache.copy_(c0)
        graph.replay()
        torch.cuda.synchronize()
        _check_select(out, _want_select(x, scores, n, None, -1), scores, None, -1)
        assert torch.equal(cache.cpu(), _moved(c0, out[1].cpu(), None))


def test_beam_sizes_are_not_cut_to_32_bits():
    ll = _ll()
    x, sc = torch.zeros((1, 2, 50), device="cuda"), torch.zeros((1, 2), device="cuda")
    ids = torch.zeros((1, 2, 4), dtype=torch.int32, device="cuda")
    for bad in (dict(n=4, end_id=(1 << 32) + 5), dict(n=(1 << 32) + 4), dict(n=4, end_id=-(1 << 40))):
        with pytest.raises(ValueError):
            ll.beam_select(x, sc, **bad)
        with pytest.raises(ValueError):
            ll.beam_merge(ids, ids.float(), sc, **bad)
    with pytest.raises(ll.LilicorrError):
        ll.beam_select(x, sc, 1 << 30)


def test_beam_reorder_refuses_states_that_share_memory():
    ll = _ll()
    parents = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    s = torch.arange(48, dtype=torch.float32, device="cuda").reshape(1, 2, 6, 4)
    keep = s.clone()
    with pytest.raises(ll.LilicorrError):
        ll.beam_reorder([s, s], parents)
    with pytest.raises(ll.LilicorrError):                      # halves of the positions, one in common
        ll.beam_reorder([s[:, :, :4], s[:, :, 2:]], parents)
    with pytest.raises(ll.LilicorrError):
        ll.beam_reorder(s[:, :1].expand(1, 2, 6, 4), parents)
    with pytest.raises(ValueError):
        ll.beam_reorder([s, s.view(torch.int32)], parents)
    assert torch.equal(s, keep)
    ll.beam_reorder([s[:, :, :2], s[:, :, 4:], s[:, :, 2:4]], parents)
    assert torch.equal(s, keep.flip(1))
