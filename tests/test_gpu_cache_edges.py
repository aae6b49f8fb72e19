"""Calls on 4-bit caches at the edges of what their contract allows, on the GPU, against plain 64-bit forms."""
import math

import pytest
import torch

import _cache_plain as plain
import test_gpu_cache as base

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------- large fp32 queries
# The scale's rest (what its rounding to fp32 left) is below 0 for d = 32, 96, 112 and 128, above for 64.
LARGE = [(32, 1, 130), (112, 9, 130), (128, 1, 3000), (96, 3, 3000), (64, 9, 3000)]


def _check_large(got, want, gain, w0, w, X, lse_tol):
    """X bounds the sum of a score's terms in size. Where a row's probabilities are taken a second time, for the weights,
    they differ by its way to log2 units: on either side four roundings of 2^-24 X (reference, its difference, the
    scale's rest, the sum)."""
    (out, lse), wlse = got, want[1]
    seen = wlse > -math.inf
    assert bool(out[seen].isfinite().all()) and bool(lse[seen].isfinite().all())
    assert bool((out[~seen] == 0).all()) and bool((lse[~seen] == -math.inf).all())
    over = (lse.double() - wlse).abs() - (2.0 ** -16 + lse_tol)
    assert bool((over[seen] <= 0).all()), float(over[seen].max())
    tol = (math.expm1(2.0 ** -21 * X) + 2.0 ** -14) * gain + 2.0 ** -22 * (w0 + gain)
    over = (w.double() - w0 - gain).abs() - tol
    assert bool((over <= 0).all()), float(over.max())


@pytest.mark.parametrize("d,T,S", LARGE)
def test_large_fp32_queries_of_one_element(d, T, S):
    """Keys of few levels along the only element that queries have: the best tie exactly and nothing else counts, so
    far scores' rounding moves no probability. lse is a reference of a score's size with four roundings (2^-24
    each) and a product with log 2 (2^-28). Lengths leave some warps without a key that a row sees."""
    ll, g, N, Hq, H = base._ll(), base._gen(d + T), 4, 8, 2
    lens = base._ints([1, 100, 129, S])
    level = torch.tensor([0.0, 1.0, 2.0, 3.0], device="cuda")
    k = torch.zeros((N, S, H, d), device="cuda")
    k[..., 0] = level[torch.randint(0, 4, (N, S, H), generator=g, device="cuda")]
    k[..., 1] = 6.0                                  # the group's largest: a scale of 1, levels exact
    v = torch.randn((N, S, H, d), generator=g, device="cuda")
    c = base._empty(N, S, H, d)
    ll.cache_append(c, k, v, torch.full_like(lens, S))
    w = torch.rand((N, H, S), generator=g, device="cuda")
    for size in (65536.0, 98304.0, 131072.0, -114688.0):
        q = torch.zeros((N, T, Hq, d), device="cuda")
        q[..., 0] = size
        w1 = w.clone()
        got = ll.cache_attention(q, c, lens, weights=w1)
        want = plain.attention(q, c, lens, d ** -0.5)
        _check_large(got, want, want[2], w, w1, 3 * abs(size) * d ** -0.5, 2.0 ** -21 * want[1].abs())
        seen = want[1] > -math.inf
        over = (got[0].double() - want[0]).abs() - (2.0 ** -15 * want[3] + 2.0 ** -23 * want[0].abs())
        assert bool((over[seen] <= 0).all()), float(over[seen].max())
        alone = ll.cache_attention(q, c, lens)
        assert torch.equal(alone[0], got[0]) and torch.equal(alone[1], got[1])


@pytest.mark.parametrize("scale", [None, 8.0e3])
@pytest.mark.parametrize("d,T,S", LARGE)
def test_large_fp32_queries(d, T, S, scale):
    """Queries of 1e4 with one element of 2e5, or of 1 at a large scale. A score's d / 16 * 3 <= 24 matrix steps round
    by at most 2^-23 X each and its way to log2 units four times by 2^-24 X: in all below 2^-18 X, and lse moves no
    more than the largest score's error does. Of the weights only the sums are told: a row gives away 1."""
    ll, g, N, Hq, H = base._ll(), base._gen(d + T), 4, 8, 2
    lens = base._ints([1, 100, 129, S])
    c = base._filled(ll, g, N, S, H, d, torch.full_like(lens, S))
    q = torch.randn((N, T, Hq, d), generator=g, device="cuda")
    if scale is None:
        q = 1e4 * q
        q[..., 5] = 2e5
    s = d ** -0.5 if scale is None else scale
    w = torch.zeros((N, H, S), device="cuda")
    got = ll.cache_attention(q, c, lens, scale=scale, weights=w)
    want = plain.attention(q, c, lens, s)
    X = s * torch.einsum("nthrd,njhd->nthrj", q.double().abs().view(N, T, H, Hq // H, d),
                         plain.values(c[..., :d // 2 + 8]).abs()).amax(4).flatten(2)
    top = float(X.max())
    assert top < 2.0 ** 20
    rows = (want[1] > -math.inf).view(N, T, H, Hq // H).sum((1, 3)).double()             # what each kv head gives away
    _check_large(got, want, rows, 0.0, w.double().sum(2), top, 2.0 ** -18 * X)

# ------------------------------------------------------------------------------- lengths past the capacity
@pytest.mark.parametrize("path", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,Hq,H,d,S", [(6, 8, 2, 64, 8), (2, 4, 1, 128, 130), (16, 32, 2, 128, 300), (70, 8, 4, 48, 64),
                                        (9, 12, 3, 32, 1500), (40, 8, 1, 80, 1300)])
def test_lengths_past_the_capacity(T, Hq, H, d, S, dtype, path):
    """Token t has position seq_len - T + t, as in cache_append, wherever the capacity ends: it sees those up to its own
    that the cache holds."""
    ll, g = base._ll(), base._gen(T + S)
    lens = base._ints([S + 1, S + T // 2, S + T - 1, S + T + 5, S, 2 ** 31 - 1])
    N = len(lens)
    was = ll.test_cache_attention_path(path)
    try:
        c = base._filled(ll, g, N, S, H, d, lens)
        q = (1.5 * torch.randn((N, T, Hq, d), generator=g, device="cuda")).to(base.DT[dtype])
        w = torch.rand((N, H, S), generator=g, device="cuda")
        w1 = w.clone()
        first = ll.cache_attention(q, c, lens)
        again = ll.cache_attention(q, c, lens, weights=w1)
    finally:
        ll.test_cache_attention_path(was)
    gain = torch.zeros((N, H, S), dtype=torch.float64, device="cuda")
    for t in range(T):                               # one token over as many positions as it sees
        ends = (lens.long() - (T - 1 - t)).clamp(0, S).int()
        base._check((first[0][:, t:t + 1], first[1][:, t:t + 1]), q[:, t:t + 1], c, ends)
        gain += plain.attention(q[:, t:t + 1], c, ends, d ** -0.5)[2]
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    over = (w1.double() - w - gain).abs() - (2.0 ** -14 * gain + 2.0 ** -22 * (w + gain))
    assert bool((over <= 0).all()), float(over.max())

# ------------------------------------------------------------------------------- records byte by byte
def _half_records(x, unit=1.0):
    """x [..., d] as half records: codes, scales, zeros up to eight of them."""
    g = x.double().unflatten(-1, (-1, 16)) / unit
    top = g.abs().amax(-1)
    scale = plain.nearest(top.clamp(max=1e300) / 6, plain.SCALES[:127]).clamp(min=1)
    s = torch.tensor(plain.SCALES, dtype=torch.float64, device=x.device)[scale]
    code = plain.nearest((g.abs() / s[..., None]).nan_to_num(0.0, posinf=9.0), plain.CODES)
    code = torch.where(top.isnan()[..., None], 0, code)          # of a NaN group, signs alone
    bits, top_bit = (torch.int32, 31) if x.dtype == torch.float32 else (torch.int16, 15)
    sign = (x.view(bits).int() >> top_bit & 1).unflatten(-1, (-1, 16))
    code = (code + 8 * sign).flatten(-2)
    scales = torch.zeros((*x.shape[:-1], 8), dtype=torch.long, device=x.device)
    scales[..., :scale.shape[-1]] = torch.where(top.isnan(), 127, scale)
    return torch.cat([code[..., ::2] + 16 * code[..., 1::2], scales], -1).byte()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 48, 80, 112, 128])
def test_records_byte_by_byte(d, dtype):
    """Codes, scales and the rest of a record are the same bytes for both types: zeros keep their sign, negative
    elements that round to zero too, and a NaN group has signs alone."""
    ll, g, N, T, H = base._ll(), base._gen(d), 3, 50, 2
    x = torch.randn((N, T, H, d // 16, 16), generator=g, device="cuda")
    pick = torch.randint(0, 8, x.shape, generator=g, device="cuda")
    for i, to in enumerate((0.0, -0.0, 2.0 ** -16, -2.0 ** -16, -2.0 ** -100)):
        x = torch.where(pick == i, torch.tensor(to, device="cuda"), x)
    x[0, 0] = -0.0
    x[0, 1, :, :, 3] = -math.inf
    x[0, 2, :, :, 5] = math.nan
    x[0, 3, :, :, 1] = -math.nan
    x = x * torch.exp2(torch.randint(-12, 8, (N, T, H, d // 16, 1), generator=g, device="cuda").float())
    x = x.flatten(3).to(base.DT[dtype]).contiguous()
    lens = base._ints([T] * N)
    for unit in (1.0, 2.0 ** -9):
        c = base._empty(N, T, H, d)
        ll.cache_append(c, x, -x, lens, k_unit=unit)
        assert torch.equal(c, torch.cat([_half_records(x, unit), _half_records(-x)], -1)), unit

# ------------------------------------------------------------------------------- eviction
def test_evict_a_shared_cache_into_others():
    """One prompt's records stand for all sequences (a stride of 0): read, they may, and each gets its own choice."""
    ll, N, S, H, d, budget = base._ll(), 3, 200, 2, 64, 50
    c, w, lens = base._evict_case(N, S, H, d, [200, 150, 40], 5)
    one = c[:1].clone()
    shared = one.expand(N, S, H, d + 16)
    want, new = plain.evict(w.cpu(), lens.tolist(), budget, 10, 2)
    to, to_w = base._empty(N, 64, H, d), torch.full((N, H, 64), 5.0, device="cuda")
    kept, new_len = ll.cache_evict(shared, w, lens, budget, recent=10, first=2, into=to, into_weights=to_w)
    assert torch.equal(kept.cpu(), want) and torch.equal(new_len.cpu(), new)
    there, at, h = kept >= 0, kept.clamp(min=0).long(), torch.arange(H, device="cuda")[:, None]
    assert torch.equal(to[:, :budget].transpose(1, 2), torch.where(there[..., None], one[0][at, h], 0x7F))
    assert base._same(to_w[..., :budget].contiguous(), torch.where(there, torch.gather(w, 2, at), 5.0))
    # written, it may not: in place, and as what is written into
    with pytest.raises(ll.LilicorrError):
        ll.cache_evict(shared, w, lens, budget)
    with pytest.raises(ll.LilicorrError):
        ll.cache_evict(c, w, lens, budget, into=shared, into_weights=w.clone())


@pytest.mark.parametrize("weights", ["spread", "ties", "nan"])
@pytest.mark.parametrize("case", [
    # N, S, H, d, lengths, budget, recent, first: on 152 SMs clusters of 4, 2, 1 CTAs an item, ...
    (10, 900, 4, 128, [900 - 37 * i for i in range(10)], 600, 50, 3),
    (20, 700, 4, 80, [700 - 30 * i for i in range(20)], 333, 20, 0),
    (100, 1300, 2, 128, [1300 - 7 * i for i in range(100)], 1000, 100, 4),
    (200, 90, 1, 16, [90 - i % 60 for i in range(200)], 44, 3, 1),
    # ... of 4 with a stretch of 2,500 each, of 2 with more than are kept in shared memory, and one CTA with as many
    (10, 10000, 4, 32, [10000 - 100 * i for i in range(10)], 700, 64, 4),
    (40, 17000, 2, 16, [17000 - 50 * i for i in range(40)], 9000, 64, 4),
    (160, 9000, 1, 16, [9000 - 10 * i for i in range(160)], 8500, 100, 2),
])
def test_evict_clusters_of_every_size(case, weights):
    base.test_evict(case, weights)


# ------------------------------------------------------------------------------- far scores
@pytest.mark.parametrize("path", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,T,S", [(64, 1, 400), (128, 4, 3000), (32, 20, 3000), (96, 9, 700)])
def test_far_scores_that_lie_close(d, T, S, dtype, path):
    """Scores of nearly 2^23, the largest that the contract has, some a few units apart, in any order: rows keep finite
    numbers. X, terms and tolerance as in test_large_fp32_queries; bf16 has a third of its matrix steps."""
    ll, g, N, Hq, H = base._ll(), base._gen(d + T), 3, 8, 2
    lens = base._ints([129, 100, S])
    k = torch.zeros((N, S, H, d), device="cuda")
    k[..., 0] = torch.tensor([2.0, 3.0], device="cuda")[(torch.rand((N, S, H), generator=g, device="cuda") < 0.7).long()]
    k[..., 1] = 6.0                                  # the group's largest: a scale of 1
    k[..., 2] = torch.randint(0, 5, (N, S, H), generator=g, device="cuda").float()       # (half steps: rounded)
    v = torch.randn((N, S, H, d), generator=g, device="cuda")
    c = base._empty(N, S, H, d)
    ll.cache_append(c, k, v, torch.full_like(lens, S))
    s = d ** -0.5
    q = torch.zeros((N, T, Hq, d), device="cuda")
    q[..., 0] = 0.98 * 2.0 ** 23 / (3 * s)
    q[..., 2] = torch.rand((N, T, Hq), generator=g, device="cuda") * 2 / s
    q = q.to(base.DT[dtype])
    was = ll.test_cache_attention_path(path)
    try:
        out, lse = ll.cache_attention(q, c, lens)
    finally:
        ll.test_cache_attention_path(was)
    want, wlse, _, _ = plain.attention(q, c, lens, s)
    X = s * (3 * q[..., 0].double() + 4 * q[..., 2].double())
    assert float(X.max()) < 2.0 ** 23
    seen = wlse > -math.inf
    assert bool(out[seen].isfinite().all()) and bool((out[~seen] == 0).all())
    assert bool((out[seen].abs().float() <= 1.01 * plain.values(c[..., d // 2 + 8:]).abs().max()).all())
    over = (lse.double() - wlse).abs() - (2.0 ** -16 + 2.0 ** -18 * X)
    assert bool((over[seen] <= 0).all()), float(over[seen].max())
    assert bool((lse[~seen] == -math.inf).all())
