"""Attention of sequences that share a prefix, against a plain 64-bit form on the keys that are there.

Tolerances. With A = sum_j p_j |v_j| (p the exact probabilities): a relative error e of every p moves
an output by at most 2 e A (it enters the sum and the normaliser). Scores here are at most 2^5 in log2
units, so each of the d <= 128 roundings of a score's fp32 sum is at most 2^-20, their sum (of either
sign, 4 sqrt(d) of the mean size 2^-21.8) below 2^-16, and ex2.approx adds 2^-22: e = 2^-16 for fp32,
so 2^-15 A, and 2^-23 of the normaliser's own size. bf16 rounds each p once more before the second
product (2^-8 of it, not of the sum: 2^-8 A) and the output (2^-8 of it)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _ll():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_20530_gb300 as ll
    return ll


def _plain(q, pk, pv, k, v, plen, slen, scale):
    """(out, lse, A) in 64 bits; rows of absent sequences are NaN."""
    N, T, Hq, d = q.shape
    G, P, Hkv, _ = pk.shape
    S, W, rep = k.shape[1], N // G, Hq // Hkv
    out = torch.full(q.shape, math.nan, dtype=torch.float64, device=q.device)
    A = out.clone()
    lse = torch.full((N, T, Hq), math.nan, dtype=torch.float64, device=q.device)
    for n in range(N):
        s1 = int(slen[n])
        if s1 < 0:
            continue
        p1, s1 = min(max(int(plen[n // W]), 0), P), min(s1, S)
        kk = torch.cat([pk[n // W, :p1], k[n, :s1]]).double().repeat_interleave(rep, 1)
        vv = torch.cat([pv[n // W, :p1], v[n, :s1]]).double().repeat_interleave(rep, 1)
        for t in range(T):
            m = p1 + max(s1 - (T - 1 - t), 0)
            s = torch.einsum("hd,jhd->hj", q[n, t].double(), kk[:m]) * scale
            lse[n, t] = torch.logsumexp(s, 1) if m else -math.inf
            p = torch.softmax(s, 1)
            out[n, t] = torch.einsum("hj,jhd->hd", p, vv[:m])
            A[n, t] = torch.einsum("hj,jhd->hd", p, vv[:m].abs())
    return out, lse, A


def _inputs(G, W, T, Hq, Hkv, d, P, S, dtype, seed, plen=None, slen=None, heads_first=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, N = DT[dtype], G * W
    if plen is None:
        plen = torch.randint(0, P + 1, (G,), generator=g, device="cuda").int()
    else:
        plen = torch.tensor(plen, dtype=torch.int32, device="cuda")
    if slen is None:
        slen = torch.randint(0, S + 1, (N,), generator=g, device="cuda").int()
    else:
        slen = torch.tensor(slen, dtype=torch.int32, device="cuda")

    def cache(B, L, lens):
        c = torch.randn((B, L, Hkv, d), generator=g, device="cuda")
        c[torch.arange(L, device="cuda")[None] >= lens[:, None]] = math.nan      # never written
        c = c.to(dt)
        return c.transpose(1, 2).contiguous().transpose(1, 2) if heads_first else c
    q = (1.5 * torch.randn((N, T, Hq, d), generator=g, device="cuda")).to(dt)
    return [q, cache(G, P, plen), cache(G, P, plen), cache(N, S, slen), cache(N, S, slen), plen, slen]


def _check(got, x, dtype, scale=None, before=None):
    q = x[0]
    scale = q.shape[3] ** -0.5 if scale is None else scale
    out, lse = got
    want, wlse, A = _plain(*x, scale)
    assert out.shape == q.shape and out.dtype == q.dtype and lse.dtype == torch.float32
    there = ~torch.isnan(wlse)
    if before is not None:                                # absent sequences: as they were
        assert torch.equal(out[~there].float(), before[0][~there].float())
        assert torch.equal(lse[~there], before[1][~there])
    out, lse, want, wlse, A = out[there].double(), lse[there].double(), want[there], wlse[there], A[there]
    empty = torch.isinf(wlse)
    assert torch.equal(torch.isinf(lse), empty) and bool((lse[empty] == -math.inf).all())
    assert bool((out[empty] == 0).all())
    out, lse, want, wlse, A = out[~empty], lse[~empty], want[~empty], wlse[~empty], A[~empty]
    if not out.numel():
        return
    assert bool(torch.isfinite(out).all())
    tol = 2.0 ** -15 * A + 2.0 ** -23 * want.abs()
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * A + 2.0 ** -8 * want.abs()
    over = (out - want).abs() - tol
    assert bool((over <= 0).all()), (float(over.max()), int((over > 0).sum()))
    over = (lse - wlse).abs() - (2.0 ** -16 + 2.0 ** -22 * wlse.abs())
    assert bool((over <= 0).all()), float(over.max())


SHAPES = [
    # G, W, T, Hq, Hkv, d, P, S
    (1, 1, 1, 1, 1, 8, 1, 1), (1, 4, 1, 8, 2, 64, 200, 24), (2, 3, 1, 4, 4, 128, 65, 64),
    (3, 5, 2, 8, 4, 96, 177, 33), (1, 1, 16, 8, 1, 128, 300, 40), (2, 4, 16, 4, 2, 64, 129, 17),
    (1, 33, 1, 8, 2, 80, 1000, 7), (2, 7, 5, 6, 2, 32, 511, 70), (1, 130, 1, 4, 2, 128, 700, 65),
    (1, 9, 3, 10, 1, 48, 1500, 129), (5, 1, 1, 16, 2, 128, 2100, 300), (1, 64, 4, 8, 2, 128, 260, 9),
    (2, 3, 1, 32, 4, 128, 1500, 600), (3, 2, 4, 8, 1, 64, 513, 530), (2, 60, 2, 16, 4, 96, 777, 40),
    (1, 2, 1, 4, 1, 128, 5000, 1100), (4, 8, 1, 8, 8, 128, 512, 64), (1, 40, 3, 8, 2, 128, 512, 7),
    (1, 300, 1, 2, 2, 64, 640, 5), (1, 129, 1, 1, 1, 128, 4000, 1), (2, 40, 8, 8, 8, 128, 130, 130),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype):
    ll = _ll()
    x = _inputs(*shape, dtype, sum(shape))
    ws = ll.Workspace(ll.prefix_attention_workspace_bytes(x[0], x[1], x[3]))
    first = ll.prefix_attention(*x, ws=ws)
    _check(first, x, dtype)
    again = ll.prefix_attention(*x, ws=ws)                 # the same workspace, the same bits
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    assert ws.status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,plen,slen", [
    (1, [0, 0], [0, 0, 0, 0]), (1, [0, 5], [1, 0, 0, 3]), (3, [0, 70], [0, 1, 2, 3]),
    (3, [0, 0], [1, 2, 0, 9]), (1, [64, 128], [64, 65, 1, 0]), (2, [63, 129], [2, 128, 130, 127]),
    (1, [-3, 500], [200, 130, 1, 2])])
def test_lengths_empty_rows_and_clipping(dtype, T, plen, slen):
    """Rows that see no key give 0 and -inf; lengths below zero and past the capacity are clipped."""
    ll = _ll()
    x = _inputs(2, 2, T, 8, 2, 64, 130, 130, dtype, 5 + T, plen, slen)
    _check(ll.prefix_attention(*x), x, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_absent_sequences_are_left_alone(dtype):
    ll = _ll()
    x = _inputs(2, 3, 2, 4, 2, 64, 90, 20, dtype, 8, [90, 0], [4, -1, 0, -1, -7, 20])
    out = torch.full_like(x[0], 7.0)
    lse = torch.full(x[0].shape[:3], 9.0, device="cuda")
    before = (out.clone(), lse.clone())
    got = ll.prefix_attention(*x, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    _check(got, x, dtype, before=before)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P,S", [(0, 40), (150, 0), (0, 0)])
def test_one_side_only(dtype, P, S):
    ll = _ll()
    x = _inputs(2, 3, 1, 4, 2, 128, P, S, dtype, 9)
    _check(ll.prefix_attention(*x), x, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 3, 2, 8, 2, 64, 140, 30), (1, 40, 1, 8, 4, 128, 333, 12),
                                   (3, 2, 1, 4, 1, 80, 270, 66)])
def test_strides(dtype, shape):
    """Caches by head, q and out cut from wider rows, a scale of the caller's."""
    ll = _ll()
    G, W, T, Hq, Hkv, d, P, S = shape
    x = _inputs(*shape, dtype, 3 + d, heads_first=True)
    wide = torch.full((G * W, T, Hq + 3, d + 16), 5.0, device="cuda", dtype=DT[dtype])
    wide[:, :, 1:Hq + 1, 8:8 + d] = x[0]
    x[0] = wide[:, :, 1:Hq + 1, 8:8 + d]
    res = torch.full((T, G * W, Hq, d + 8), 3.0, device="cuda", dtype=DT[dtype])
    out = res.transpose(0, 1)[..., :d]
    _check(ll.prefix_attention(*x, scale=0.05, out=out), x, dtype, scale=0.05)
    assert bool((res[..., d:] == 3.0).all())
    # one prefix for all groups, by a stride of zero
    one = [x[0], x[1][:1].expand(G, -1, -1, -1), x[2][:1].expand(G, -1, -1, -1), *x[3:]]
    one[5] = x[5][:1].expand(G).contiguous()
    _check(ll.prefix_attention(*one), one, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores_and_equal_scores(dtype):
    """One key far ahead of the others late in the prefix (the running maximum moves), and constant
    keys (plain means)."""
    ll = _ll()
    x = _inputs(1, 3, 1, 4, 2, 64, 700, 80, dtype, 21, [700], [80, 40, 1])
    x[1][0, 650] = 4 * x[0][0, 0, 0]
    x[3][1, 20] = -3 * x[0][1, 0, 1]
    _check(ll.prefix_attention(*x, scale=0.02), x, dtype, scale=0.02)
    y = list(x)
    y[1], y[3] = torch.ones_like(x[1]), torch.ones_like(x[3])
    _check(ll.prefix_attention(*y), y, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(dtype):
    """A cache whose second group lies more than 2^31 elements behind the first."""
    ll = _ll()
    x = _inputs(2, 2, 1, 4, 2, 64, 200, 30, dtype, 31, [200, 150], [30, 7, 1, 12])
    es = x[0].element_size()
    far = (1 << 31) + 4096
    big = torch.empty(far + x[1][0].numel(), dtype=DT[dtype], device="cuda")
    view = torch.as_strided(big, x[1].shape, (far,) + x[1].stride()[1:])
    view.copy_(x[1])
    assert (view.data_ptr() + far * es) - view.data_ptr() > 1 << 32
    _check(ll.prefix_attention(x[0], view, *x[2:]), x, dtype)
    view.copy_(x[2])
    _check(ll.prefix_attention(x[0], x[1], view, *x[3:]), x, dtype)
    del big, view


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_replayed_and_on_another_stream(dtype):
    """Captured once, replayed with other lengths and contents; two graphs with a workspace each."""
    ll = _ll()
    shape = (2, 4, 1, 8, 2, 64, 600, 40)
    x = _inputs(*shape, dtype, 1)
    st = torch.cuda.Stream()
    outs, graphs = [], []
    for _ in range(2):
        ws = ll.Workspace(ll.prefix_attention_workspace_bytes(x[0], x[1], x[3]))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            outs.append(ll.prefix_attention(*x, ws=ws) + (ws,))
        graphs.append(graph)
    for seed in (2, 3):
        for a, b in zip(x, _inputs(*shape, dtype, seed)):
            a.copy_(b)
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for o in outs:
            _check(o[:2], x, dtype)
            assert o[2].status() == 0


@pytest.fixture(params=[1, 2])
def path(request):
    """Both kernels of a bf16 prefix, whatever the sizes."""
    ll = _ll()
    prev = ll.test_prefix_path(request.param)
    yield request.param
    ll.test_prefix_path(prev)


@pytest.mark.parametrize("shape", SHAPES)
def test_shapes_on_both_paths(shape, path):
    test_shapes(shape, "bf16")


@pytest.mark.parametrize("T,plen,slen", [
    (1, [0, 0], [0, 0, 0, 0]), (1, [0, 5], [1, 0, 0, 3]), (3, [0, 70], [0, 1, 2, 3]),
    (3, [0, 0], [1, 2, 0, 9]), (1, [64, 128], [64, 65, 1, 0]), (2, [63, 129], [2, 128, 130, 127]),
    (1, [-3, 500], [200, 130, 1, 2])])
def test_lengths_on_both_paths(T, plen, slen, path):
    test_lengths_empty_rows_and_clipping("bf16", T, plen, slen)


def test_layouts_on_both_paths(path):
    """Absent sequences, one side only, strides, large scores, far groups, graphs."""
    test_absent_sequences_are_left_alone("bf16")
    test_one_side_only("bf16", 150, 0)
    for shape in ((2, 3, 2, 8, 2, 64, 140, 30), (1, 40, 1, 8, 4, 128, 333, 12), (3, 2, 1, 4, 1, 80, 270, 66)):
        test_strides("bf16", shape)
    test_large_scores_and_equal_scores("bf16")
    test_offsets_past_32_bits("bf16")
    test_captured_replayed_and_on_another_stream("bf16")


def test_many_groups_on_both_paths(path):
    """More groups than a CTA has threads, some without a prefix: the list of tiles is cut inside and between
    them."""
    ll = _ll()
    G = 800
    x = _inputs(G, 1, 1, 2, 1, 64, 200, 3, "bf16", 11, [(37 * g) % 201 if g % 5 else 0 for g in range(G)])
    _check(ll.prefix_attention(*x), x, "bf16")


@pytest.mark.parametrize("P,S", [(512, 256), (512, 257), (513, 16), (64, 385), (0, 384), (0, 385)])
@pytest.mark.parametrize("W", [2, 90])
def test_sides_of_the_plan(P, S, W):
    """Capacities on both sides of where a prefix goes in front of the own keys, and pieces begin."""
    ll = _ll()
    x = _inputs(1, W, 1, 8, 2, 64, P, S, "bf16", P + S + W)
    _check(ll.prefix_attention(*x), x, "bf16")


def test_two_streams_at_once():
    ll = _ll()
    xs = [_inputs(2, 8, 1, 8, 2, 128, 3000, 60, "bf16", s) for s in (1, 2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    wss = [ll.Workspace(ll.prefix_attention_workspace_bytes(x[0], x[1], x[3])) for x in xs]
    torch.cuda.synchronize()
    outs = [None, None]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                outs[i] = ll.prefix_attention(*xs[i], ws=wss[i])
    torch.cuda.synchronize()
    for o, x in zip(outs, xs):
        _check(o, x, "bf16")


@pytest.mark.parametrize("which", [1, 2])
@pytest.mark.parametrize("W", [3, 70])
def test_bounded_waits_run_out(which, W):
    """The tensor-core kernel without its K or its V copies: it records the timeout, and the context and
    the workspace are as good as before."""
    ll = _ll()
    x = _inputs(2, W, 1, 8, 2, 64, 700, 8, "bf16", 3, [700, 530], [4] * (2 * W))
    ws = ll.Workspace(ll.prefix_attention_workspace_bytes(x[0], x[1], x[3]))
    ll.test_prefix_attention_timeout(*x, ws, 2_000_000, which)
    assert ws.status() == 6
    _check(ll.prefix_attention(*x, ws=ws), x, "bf16")
    assert ws.status() == 0


def test_python_refusals():
    ll = _ll()
    x = _inputs(2, 2, 1, 4, 2, 64, 20, 10, "bf16", 1)
    for i, bad in ((0, x[0].float()), (0, x[0].cpu()), (0, x[0][:3]), (1, x[1].transpose(2, 3)),
                   (2, x[2][:, :19]), (4, x[4].float()), (5, x[5].long()), (6, x[6][:3]),
                   (0, x[0][0]), (3, x[3].half())):
        y = list(x)
        y[i] = bad
        with pytest.raises(ValueError):
            ll.prefix_attention(*y)
    for kw in (dict(scale=0.0), dict(scale=math.inf), dict(scale=-1.0), dict(ws=ll.Workspace(256))):
        with pytest.raises(ll.LilicorrError):
            ll.prefix_attention(*x, **kw)
    odd = torch.empty((4, 1, 4, 65), dtype=torch.bfloat16, device="cuda")[..., :64]    # rows of 130 bytes
    with pytest.raises(ll.LilicorrError):
        ll.prefix_attention(odd, *x[1:])
    with pytest.raises(ll.LilicorrError):
        ll.prefix_attention(*(c[..., :60].contiguous() for c in x[:5]), *x[5:])        # d % 8


def test_a_beam_search_decodes_as_its_plain_form():
    """Six steps of beam search of a small attention model on two requests: attention behind the
    shared prompt, logits, beam_select and beam_reorder of the beams' caches, against the same steps in
    64 bits. Greedy in their gaps: the plain form follows the kernel's picks after checking them."""
    ll = _ll()
    g = torch.Generator(device="cuda").manual_seed(0)
    R, W, Hq, Hkv, d, P, V, steps = 2, 3, 4, 2, 32, 50, 211, 6
    H = Hq * d
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    emb, wq, wk, wv, wl = rn(V, H), rn(H, H) / H ** .5, rn(H, Hkv * d) / H ** .5, \
        rn(H, Hkv * d) / H ** .5, rn(H, V) * 3 / H ** .5
    pk, pv = rn(R, P, Hkv, d), rn(R, P, Hkv, d)
    plen = torch.tensor([P, 31], dtype=torch.int32, device="cuda")
    k, v = torch.full((R * W, steps, Hkv, d), math.nan, device="cuda"), \
        torch.full((R * W, steps, Hkv, d), math.nan, device="cuda")
    tokens = torch.tensor([[1, 0, 0], [2, 0, 0]], dtype=torch.int32, device="cuda")
    scores = torch.tensor([[0.0, -math.inf, -math.inf]] * 2, device="cuda")
    done = torch.zeros((R, W), dtype=torch.bool, device="cuda")
    end = 5
    hist = [[[] for _ in range(W)] for _ in range(R)]        # each beam's tokens
    exact = torch.tensor([[0.0, -math.inf, -math.inf]] * 2, dtype=torch.float64)
    for step in range(steps):
        h = emb[tokens.clamp(min=0).long()].view(R * W, H)
        k[:, step] = (h @ wk).view(R * W, Hkv, d)
        v[:, step] = (h @ wv).view(R * W, Hkv, d)
        slen = torch.full((R * W,), step + 1, dtype=torch.int32, device="cuda")
        o, _ = ll.prefix_attention((h @ wq).view(R * W, 1, Hq, d), pk, pv, k, v, plen, slen)
        logits = ((o.view(R * W, H) + h) @ wl).view(R, W, V)
        was_done, was = done.cpu(), tokens.cpu()
        tokens, parents, scores, done = ll.beam_select(logits.contiguous(), scores, W, done=done,
                                                       end_id=end)
        ll.beam_reorder([k.view(R, W, steps, Hkv, d), v.view(R, W, steps, Hkv, d)], parents,
                        torch.full((R,), step + 1, dtype=torch.int32, device="cuda"))
        # the same step in 64 bits, from each beam's own tokens
        total = torch.full((R, W, V), -math.inf, dtype=torch.float64)
        for r in range(R):
            for w in range(W):
                if exact[r, w] == -math.inf:
                    continue
                if was_done[r, w]:
                    total[r, w, end] = exact[r, w]
                    continue
                seq = hist[r][w] + [int(was[r, w])]
                hh = emb[seq].double()
                kk = torch.cat([pk[r, :plen[r]].double(), (hh @ wk.double()).view(-1, Hkv, d)])
                vv = torch.cat([pv[r, :plen[r]].double(), (hh @ wv.double()).view(-1, Hkv, d)])
                qq = (hh[-1] @ wq.double()).view(Hkv, Hq // Hkv, d)
                p = torch.softmax(torch.einsum("grd,jgd->grj", qq, kk) * d ** -0.5, 2)
                at = torch.einsum("grj,jgd->grd", p, vv).reshape(H)
                total[r, w] = exact[r, w] + torch.log_softmax((at + hh[-1]) @ wl.double(), 0).cpu()
        new_hist, new_exact = [[None] * W for _ in range(R)], torch.empty_like(exact)
        for r in range(R):
            order = torch.sort(total[r].flatten(), descending=True)[0]
            for j in range(W):
                pj, tj = int(parents[r, j]), int(tokens[r, j])
                # fp32 products of 128 terms: 1e-4 covers their rounding through both layers
                assert abs(float(total[r, pj, tj]) - float(order[j])) < 1e-4
                assert abs(float(scores[r, j]) - float(total[r, pj, tj])) < 1e-4
                new_exact[r, j] = total[r, pj, tj]
                new_hist[r][j] = hist[r][pj] + [int(was[r, pj])]
                assert bool(done[r, j]) == (bool(was_done[r, pj]) or tj == end)
            assert len({(int(parents[r, j]), int(tokens[r, j])) for j in range(W)}) == W
        hist, exact = new_hist, new_exact


def test_drafted_blocks_verified_behind_one_cache():
    """The greedy walk's and the best path's blocks of each request, 8 tokens each, verified behind
    the request's cache: each token's row equals the row of decoding it alone."""
    ll = _ll()
    x = _inputs(3, 2, 8, 8, 2, 64, 210, 20, "bf16", 44, [210, 64, 0], [8, 8, 12, 20, 8, 9])
    both = ll.prefix_attention(*x)
    _check(both, x, "bf16")
    for t in (0, 3, 7):
        y = list(x)
        y[0] = x[0][:, t:t + 1]
        y[6] = x[6] - (7 - t)
        one = ll.prefix_attention(*y)
        want, wlse, A = _plain(*y, 64 ** -0.5)
        # two roundings of each kind apart
        assert bool(((one[0] - both[0][:, t:t + 1]).abs() <= 2.0 ** -6 * A + 2.0 ** -7 * want.abs()).all())
