"""A decoding cache held in 4 bits on the GPU, against plain 64-bit forms.

Rounding into the cache and eviction are exact: codes, scales and positions have one right value. Attention's
tolerances: with A = sum_j p_j |v_j| (p the exact probabilities) a relative error e of every p moves an
output by at most 2 e A (it enters the sum and the normaliser). Scores here are at most 2^5 in log2 units, and
products are exact, so each of the d / 16 <= 8 matrix steps of a score (24 in fp32) rounds its sum by at
most 2^-18 (2^-23 of 2^5), in sum below 2^-15 for bf16 and 2^-14 for fp32 at worst, and ex2.approx adds 2^-22.
Steps round independently, so a quarter of the worst case is not reached: e = 2^-16. An fp32 result is
so within 2^-15 A, and 2^-23 of its own size; bf16 queries round each p to fp16 once before the second
product (2^-11 of it, and of the sums' largest 2^-24 absolutely: 2^-10 A covers both sides of the quotient) and
the output once (2^-8 of it). A position's weight is a sum of p: 2^-14 of what it gains, and 2^-22 of itself."""
import math

import pytest
import torch

import _cache_plain as plain

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _ll():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_20530_gb300 as ll
    return ll


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _empty(N, S, H, d, heads_first=False, pad=0, fill=0x7F):
    """A cache that nobody has written, records of any bytes; `pad`: 16-byte pieces between records."""
    shape = (N, H, S, d + 16 + 16 * pad) if heads_first else (N, S, H, d + 16 + 16 * pad)
    c = torch.full(shape, fill, dtype=torch.uint8, device="cuda")[..., :d + 16]
    return c.transpose(1, 2) if heads_first else c


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _filled(ll, g, N, S, H, d, lens, heads_first=False, k_unit=1.0, v_unit=1.0, fill=0x7F):
    """A cache of random keys and values, filled to its lengths by cache_append."""
    c = _empty(N, S, H, d, heads_first, fill=fill)
    k = torch.randn((N, S, H, d), generator=g, device="cuda") * k_unit
    v = torch.randn((N, S, H, d), generator=g, device="cuda") * v_unit
    ll.cache_append(c, k, v, lens.clamp(max=S), k_unit=k_unit, v_unit=v_unit)
    return c


# ------------------------------------------------------------------------------- append and read
SHAPES = [(1, 1, 1, 1, 16), (2, 3, 9, 2, 32), (3, 40, 30, 2, 80), (1, 130, 200, 8, 128), (5, 7, 64, 3, 96),
          (2, 17, 40, 1, 48), (1, 33, 33, 5, 112), (4, 9, 20, 2, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_append_and_read(shape, heads_first, dtype):
    ll, (N, T, S, H, d) = _ll(), shape
    g = _gen(sum(shape))
    size = torch.exp2(torch.randint(-14, 10, (N, T, H, d // 16, 1), generator=g, device="cuda").float())
    new = [(torch.randn((N, T, H, d // 16, 16), generator=g, device="cuda") * size).flatten(3).to(DT[dtype])
           for _ in range(2)]
    lens = torch.randint(0, S + 1, (N,), generator=g, device="cuda").int()
    lens[0] = S
    if N > 2:
        lens[1] = -1
    c = _empty(N, S, H, d, heads_first, pad=1, fill=0xA5)
    w = torch.rand((N, H, S), generator=g, device="cuda")
    before, w0 = c.clone(), w.clone()
    assert ll.cache_append(c, *new, lens, weights=w) is c
    back = ll.cache_read(c, lens, T, dtype=DT[dtype])
    pos = lens[:, None] - T + torch.arange(T, device="cuda")
    ok = (pos >= 0) & (pos < S) & (lens[:, None] >= 0)
    half = d // 2 + 8
    for x, y, part in ((new[0], back[0], slice(0, half)), (new[1], back[1], slice(half, None))):
        want = torch.where(ok[:, :, None, None], plain.round_values(x), 0.0)
        assert torch.equal(y.double(), want)
        n, t = torch.nonzero(ok, as_tuple=True)
        assert torch.equal(plain.values(c[n, pos[n, t]][..., part]), want[n, t])
    # the other positions, their weights and the space between records: as they were
    touched = torch.zeros((N, S), dtype=torch.bool, device="cuda")
    n, t = torch.nonzero(ok, as_tuple=True)
    touched[n, pos[n, t]] = True
    assert torch.equal(c[~touched], before[~touched])
    at = touched[:, None, :].expand(N, H, S)
    assert bool((w[at] == 0).all()) and torch.equal(w[~at], w0[~at])
    whole = c._base if c._base is not None else c
    assert bool((whole[..., d + 16:] == 0xA5).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_borders_between_values(dtype):
    """Every scale, every border between two codes, and its neighbours on either side."""
    ll = _ll()
    rows = []
    for s in plain.SCALES[1:127]:
        row = [6 * s]
        for m in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
            row += [m * s, -m * s]
        rows.append(row + [0.0])
    x = torch.tensor(rows, dtype=torch.float64, device="cuda").to(DT[dtype])
    step = torch.finfo(DT[dtype]).eps
    x = torch.cat([x, x * (1 + step), x * (1 - step)])
    # and the borders between two scales
    s = torch.tensor(plain.SCALES[1:127], dtype=torch.float64, device="cuda")
    mid = (6 * (s[1:] + s[:-1]) / 2).to(DT[dtype])
    edge = torch.cat([mid, mid * (1 + step), mid * (1 - step)])[:, None] * torch.linspace(
        0, 1, 16, device="cuda").to(DT[dtype])
    x = torch.cat([x, edge])[:, None, None, :].contiguous()
    lens = torch.ones(x.shape[0], dtype=torch.int32, device="cuda")
    c = _empty(x.shape[0], 1, 1, 16)
    ll.cache_append(c, x, -x, lens)
    k, v = ll.cache_read(c, lens, 1, dtype=DT[dtype])
    assert torch.equal(k.double(), plain.round_values(x))
    assert torch.equal(v, -k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_extremes(dtype):
    """Zeros, tiny and huge values, infinities and NaN, and what units do about them."""
    ll = _ll()
    big, tiny = torch.finfo(DT[dtype]).max, torch.finfo(DT[dtype]).tiny
    rows = [[0.0] * 16, [-0.0] * 16, [tiny] * 16, [big] + [1.0] * 15, [math.inf] + [2700.0, -1.0] + [0.5] * 13,
            [-math.inf] * 16, [math.nan] + [1.0] * 15, [2688.0] * 16, [3000.0] * 16, [2.0 ** -10] * 16,
            [2.0 ** -11] * 16, [0.01] * 16]
    x = torch.tensor(rows, dtype=torch.float64, device="cuda").to(DT[dtype])[:, None, None, :].contiguous()
    lens = torch.ones(len(rows), dtype=torch.int32, device="cuda")
    for unit in (1.0, 2.0 ** -20, 2.0 ** 40, 2.0 ** -60, 2.0 ** 60):
        c = _empty(len(rows), 1, 1, 16)
        ll.cache_append(c, x, x, lens, k_unit=unit)
        k, v = ll.cache_read(c, lens, 1, dtype=DT[dtype], k_unit=unit)
        want = plain.round_values(x, unit)
        assert torch.equal(k.double().nan_to_num(7e77), want.nan_to_num(7e77)), unit
        assert torch.equal(v.double().nan_to_num(7e77), plain.round_values(x).nan_to_num(7e77))


def test_append_views_and_short_lengths():
    """k and v may be slices of one projection; tokens outside the cache are left out."""
    ll = _ll()
    g = _gen(3)
    kv = torch.randn((4, 6, 2, 3, 32), generator=g, device="cuda").bfloat16()     # N, T, (k, v), H, d
    k, v = kv[:, :, 0], kv[:, :, 1]
    lens = _ints([6, 2, 12, 0])                      # the third one runs past the capacity of 8
    c = _empty(4, 8, 3, 32)
    before = c.clone()
    ll.cache_append(c, k, v, lens)
    got = ll.cache_read(c, lens, 6)
    want = plain.round_values(k)
    want[1, :4], want[2, 2:], want[3] = 0, 0, 0
    assert torch.equal(got[0].double(), want)
    assert torch.equal(c[0, 6:], before[0, 6:]) and torch.equal(c[3], before[3])
    assert torch.equal(c[2, :6], before[2, :6]) and not torch.equal(c[2, 6:], before[2, 6:])


# ------------------------------------------------------------------------------- attention
def _check(got, q, c, lens, scale=None, w0=None, w=None, before=None, **units):
    dtype = q.dtype
    scale = q.shape[3] ** -0.5 if scale is None else scale
    out, lse = got
    want, wlse, gain, A = plain.attention(q, c, lens, scale, **units)
    assert out.shape == q.shape and out.dtype == dtype and lse.dtype == torch.float32
    there = ~wlse.isnan()
    if before is not None:
        assert torch.equal(out[~there].float(), before[0][~there].float())
        assert torch.equal(lse[~there], before[1][~there])
    if w is not None:
        live = torch.arange(c.shape[1], device="cuda") < lens[:, None, None]
        live = live.expand_as(w)
        assert torch.equal(w[~live], w0[~live])
        over = (w[live].double() - w0[live].double() - gain[live]).abs() - (
            2.0 ** -14 * gain[live] + 2.0 ** -22 * (w0[live].abs().double() + gain[live]))
        assert not over.numel() or float(over.max()) <= 0, float(over.max())
    out, lse, want, wlse, A = out[there].double(), lse[there].double(), want[there], wlse[there], A[there]
    empty = torch.isinf(wlse)
    assert bool((lse[empty] == -math.inf).all()) and bool((out[empty] == 0).all())
    out, lse, want, wlse, A = out[~empty], lse[~empty], want[~empty], wlse[~empty], A[~empty]
    if not out.numel():
        return
    tol = 2.0 ** -15 * A + 2.0 ** -23 * want.abs()
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -10 * A + 2.0 ** -8 * want.abs()
    over = (out - want).abs() - tol
    assert bool((over <= 0).all()), (float(over.max()), int((over > 0).sum()))
    over = (lse - wlse).abs() - (2.0 ** -16 + 2.0 ** -22 * wlse.abs())
    assert bool((over <= 0).all()), float(over.max())


def _case(ll, N, T, Hq, H, d, S, dtype, seed, lens=None, heads_first=False, fill=0x7F, **units):
    g = _gen(seed)
    if lens is None:
        lens = torch.randint(0, S + 1, (N,), generator=g, device="cuda").int()
        lens[0] = S
    else:
        lens = _ints(lens)
    c = _filled(ll, g, N, S, H, d, lens, heads_first, fill=fill, **units)
    q = (1.5 * torch.randn((N, T, Hq, d), generator=g, device="cuda")).to(DT[dtype])
    w = torch.rand((N, H, S), generator=g, device="cuda")
    return q, c, lens, w


ATTENTION = [
    # N, T, Hq, H, d, S
    (1, 1, 1, 1, 16, 1), (1, 1, 8, 2, 64, 224), (2, 1, 32, 8, 128, 300), (3, 2, 8, 4, 96, 177),
    (1, 16, 8, 1, 128, 300), (2, 5, 6, 2, 32, 511), (5, 1, 5, 5, 80, 129), (1, 1, 8, 1, 48, 4000),
    (4, 3, 6, 1, 112, 700), (2, 16, 32, 4, 128, 1025), (1, 1, 16, 1, 128, 9000), (33, 1, 4, 1, 64, 257),
    (1, 40, 4, 2, 128, 65), (2, 1, 24, 1, 128, 515), (3, 7, 9, 3, 16, 50), (1, 100, 8, 1, 64, 333),
    (70, 1, 8, 8, 128, 40), (1, 1, 32, 8, 128, 20000), (2, 4, 64, 2, 128, 640), (6, 1, 12, 4, 32, 2222),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ATTENTION)
def test_attention(shape, dtype):
    ll = _ll()
    seed = sum(shape)
    q, c, lens, w = _case(ll, *shape, dtype, seed, heads_first=seed % 2 == 0)
    ws = ll.Workspace(ll.cache_attention_workspace_bytes(q, c))
    first = ll.cache_attention(q, c, lens, ws=ws)
    _check(first, q, c, lens)
    w1 = w.clone()
    again = ll.cache_attention(q, c, lens, weights=w1, ws=ws)
    _check(again, q, c, lens, w0=w, w=w1)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    w2 = w.clone()                                   # the same call, the same bits
    ll.cache_attention(q, c, lens, weights=w2, ws=ws)
    assert torch.equal(w1, w2) and ws.status() == 0


@pytest.fixture
def tensor_cores():
    """bf16 queries on the kernel that takes many rows, however few there are."""
    ll = _ll()
    was = ll.test_cache_attention_path(1)
    yield ll
    ll.test_cache_attention_path(was)


@pytest.mark.parametrize("shape", ATTENTION + [
    (1, 16, 32, 2, 128, 2000), (2, 33, 8, 1, 64, 1300), (3, 8, 32, 8, 96, 5000), (1, 130, 4, 2, 32, 260),
    (40, 4, 16, 4, 128, 700), (2, 20, 16, 1, 80, 390), (1, 64, 8, 4, 128, 9000)])
def test_attention_on_tensor_cores(tensor_cores, shape):
    ll, seed = tensor_cores, sum(shape)
    q, c, lens, w = _case(ll, *shape, "bf16", seed, heads_first=seed % 2 == 0)
    ws = ll.Workspace(ll.cache_attention_workspace_bytes(q, c))
    first = ll.cache_attention(q, c, lens, ws=ws)
    assert ws.status() == 0
    _check(first, q, c, lens)
    w1 = w.clone()
    again = ll.cache_attention(q, c, lens, weights=w1, ws=ws)
    _check(again, q, c, lens, w0=w, w=w1)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1]) and ws.status() == 0


def test_far_scores_on_tensor_cores(tensor_cores):
    """References that move at every step, queries of any size, and a row of NaN."""
    test_units_scale_and_far_scores("bf16")
    for T in (1, 3):
        test_nan_query_spoils_its_own_row("bf16", T)


@pytest.mark.parametrize("which", [1, 2, 3])
def test_bounded_waits_run_out(tensor_cores, which):
    """Products whose keys or values never come: the waits end, the status says so, the context lives."""
    ll = tensor_cores
    q, c, lens, _ = _case(ll, 2, 16, 8, 2, 128, 700, "bf16", 3)
    ws = ll.Workspace(ll.cache_attention_workspace_bytes(q, c))
    ll.test_cache_attention_timeout(q, c, lens, ws, 2_000_000, which)
    assert ws.status() == 6
    ws = ll.Workspace(ll.cache_attention_workspace_bytes(q, c))
    w = torch.zeros((2, 2, 700), device="cuda")
    w1 = w.clone()
    _check(ll.cache_attention(q, c, lens, weights=w1, ws=ws), q, c, lens, w0=w, w=w1)
    assert ws.status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,lens", [(1, [0, 1, 2]), (3, [0, 1, 2, 3, 4]), (5, [4, 70, 64, 65, 63]),
                                    (1, [500, 130, 129, 128, 127]), (2, [-3, 5, -1, 0, 130]),
                                    (16, [8, 16, 17, 15, 130])])
@pytest.mark.parametrize("path", [0, 1])
def test_lengths(dtype, T, lens, path):
    """Empty rows, absent sequences, lengths past the capacity; nothing behind a length is looked at."""
    ll = _ll()
    was = ll.test_cache_attention_path(path)
    try:
        _lengths(ll, dtype, T, lens)
    finally:
        ll.test_cache_attention_path(was)


def _lengths(ll, dtype, T, lens):
    q, c, lens, w = _case(ll, len(lens), T, 8, 2, 64, 130, dtype, T, lens, fill=0xFF)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:3], 7.0, device="cuda")
    w1 = w.clone()
    got = ll.cache_attention(q, c, lens, weights=w1, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    _check(got, q, c, lens, w0=w, w=w1, before=(torch.full_like(out, 7.0), torch.full_like(lse, 7.0)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_units_scale_and_far_scores(dtype):
    ll = _ll()
    q, c, lens, w = _case(ll, 2, 2, 4, 2, 128, 200, dtype, 4, k_unit=2.0 ** -9, v_unit=2.0 ** 12)
    w1 = w.clone()
    got = ll.cache_attention(q, c, lens, scale=30.0, weights=w1, k_unit=2.0 ** -9, v_unit=2.0 ** 12)
    _check(got, q, c, lens, 30.0, w0=w, w=w1, k_unit=2.0 ** -9, v_unit=2.0 ** 12)
    # queries of any size: a row's own power of two takes them
    for size in (2.0 ** -60, 2.0 ** 60):
        _check(ll.cache_attention(q * size, c, lens, scale=0.1 / size), q * size, c, lens, 0.1 / size)
    # keys in ascending order of their scores: every step finds a larger one
    ramp = torch.zeros((1, 300, 1, 32), device="cuda")
    ramp[0, :, 0, 0] = torch.arange(300, device="cuda").float()
    x = _empty(1, 300, 1, 32)
    full = _ints([300])
    ll.cache_append(x, ramp, torch.randn(1, 300, 1, 32, generator=_gen(1), device="cuda"), full)
    one = torch.zeros((1, 1, 2, 32), device="cuda").to(DT[dtype])
    one[..., 0] = 1.0
    for scale in (0.01, 0.1):
        _check(ll.cache_attention(one, x, full, scale=scale), one, x, full, scale)
        _check(ll.cache_attention(-one, x, full, scale=scale), -one, x, full, scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 3])
def test_nan_query_spoils_its_own_row(dtype, T):
    ll = _ll()
    q, c, lens, w = _case(ll, 2, T, 8, 2, 64, 700, dtype, 9)
    clean = ll.cache_attention(q, c, lens)
    bad = q.clone()
    bad[1, T - 1, 2, 5] = math.nan
    w1 = w.clone()
    out, lse = ll.cache_attention(bad, c, lens, weights=w1)
    spoilt = torch.zeros(q.shape[:3], dtype=torch.bool, device="cuda")
    spoilt[1, T - 1, 2] = True
    assert bool(out[spoilt].isnan().all()) and bool(lse[spoilt].isnan().all())
    assert torch.equal(out[~spoilt], clean[0][~spoilt]) and torch.equal(lse[~spoilt], clean[1][~spoilt])
    _check((out[:1], lse[:1]), bad[:1], c[:1], lens[:1], w0=w[:1], w=w1[:1])
    want = plain.attention(bad, c, lens, 64 ** -0.5)[2]
    assert bool(((w1.double() - w.double() - want).abs() <= 2.0 ** -14 * want + 2.0 ** -22 * (1 + want)).all())


@pytest.mark.parametrize("shape", [
    (40, 9, 8, 2, 96, 700), (3, 16, 32, 8, 128, 5000), (1, 16, 32, 4, 64, 9000), (2, 70, 16, 2, 128, 900),
    (300, 5, 32, 8, 128, 130), (2, 17, 1, 1, 16, 20), (5, 33, 12, 3, 48, 400), (1, 129, 2, 1, 80, 1000)])
def test_weights_of_many_rows(shape):
    """More rows a kv head than scores are kept for: one block of rows and several, items that begin and end
    anywhere in a CTA's share."""
    ll = _ll()
    q, c, lens, w = _case(ll, *shape, "bf16", 77, heads_first=shape[0] % 2 == 0)
    w1, w2 = w.clone(), w.clone()
    _check(ll.cache_attention(q, c, lens, weights=w1), q, c, lens, w0=w, w=w1)
    ll.cache_attention(q, c, lens, weights=w2)
    assert torch.equal(w1, w2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 9, 40])
def test_keys_that_are_not_finite_add_nothing(dtype, T):
    """Rows that meet such a key have no finite sum; the other kv heads and sequences do not see it."""
    ll = _ll()
    q, c, lens, w = _case(ll, 2, T, 8, 2, 64, 700, dtype, 10, lens=[700, 650])
    w1, w2 = w.clone(), w.clone()
    ll.cache_attention(q, c, lens, weights=w1)
    c[1, 300, 0, 32:40] = 0x7F                       # a key's scales: NaN
    out, lse = ll.cache_attention(q, c, lens, weights=w2)
    assert bool(out[1, :, :4].isnan().all()) and bool(lse[1, :, :4].isnan().all())
    assert torch.equal(w2[1, 0], w[1, 0])
    assert torch.equal(w2[0], w1[0]) and torch.equal(w2[1, 1], w1[1, 1])
    assert bool(out[1, :, 4:].isfinite().all()) and bool(out[0].isfinite().all())


@pytest.mark.parametrize("T", [1, 16])
def test_one_large_weight_and_very_many_small_ones(T):
    """Half of a row's weight on one key, the rest on 2^19 others: what the second product's operand loses of each
    small one it loses of all of them."""
    ll = _ll()
    S, d = (1 << 19) + 77, 16
    c = _empty(1, S, 1, d, fill=0)
    c[..., d // 2] = 0x38                            # a scale of 1, elements 0
    c[..., d + 8] = 0x38
    g = _gen(5)
    c[..., d // 2 + 8:d + 8] = torch.randint(0, 256, (1, S, 1, d // 2), generator=g, device="cuda").byte()
    c[0, 12345, 0, 0] = 0x07                         # one key of 6 along the first element
    q = torch.zeros((1, T, 4, d), device="cuda").bfloat16()
    q[..., 0] = torch.linspace(2.1, 2.3, 4, device="cuda")     # exp(6 * 2.2) = 2^19
    lens = _ints([S])
    w = torch.zeros((1, 1, S), device="cuda")
    w1 = w.clone()
    _check(ll.cache_attention(q, c, lens, scale=1.0, weights=w1), q, c, lens, 1.0, w0=w, w=w1)


def test_one_workspace_for_calls_of_any_shapes():
    """Calls that leave other parts of it written, between calls that need their counts at 0."""
    ll = _ll()
    shapes = [(1, 1, 16, 1, 128, 9000), (2, 1, 8, 2, 64, 224), (1, 1, 32, 8, 128, 20000), (2, 16, 32, 4, 128, 1025),
              (33, 1, 4, 1, 64, 257), (6, 1, 12, 4, 32, 2222)]
    cases = [_case(ll, *s, "bf16", i) for i, s in enumerate(shapes)]
    ws = ll.Workspace(max(ll.cache_attention_workspace_bytes(q, c) for q, c, _, _ in cases))
    for _ in range(2):
        for q, c, lens, w in cases:
            w1 = w.clone()
            _check(ll.cache_attention(q, c, lens, weights=w1, ws=ws), q, c, lens, w0=w, w=w1)


def test_caches_without_room():
    """A capacity of 0: nothing is written, rows see nothing, nothing is evicted."""
    ll = _ll()
    c, w = _empty(2, 0, 2, 32), torch.zeros((2, 2, 0), device="cuda")
    lens = _ints([0, 3])
    k = torch.ones((2, 1, 2, 32), device="cuda").bfloat16()
    ll.cache_append(c, k, k, lens, weights=w)
    assert bool((ll.cache_read(c, lens, 1)[0] == 0).all())
    for T in (1, 40):
        q = torch.ones((2, T, 4, 32), device="cuda").bfloat16()
        out, lse = ll.cache_attention(q, c, lens, weights=w)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    kept, new = ll.cache_evict(c, w, lens, 3)
    assert bool((kept == -1).all()) and new.tolist() == [0, 0]


def test_shared_and_strided_caches():
    """Every sequence the same cache (a stride of 0), records with space between them, strided q and out."""
    ll = _ll()
    g = _gen(6)
    lens = _ints([50])
    c = _filled(ll, g, 1, 64, 2, 48, lens)
    many = c.expand(5, 64, 2, 64)
    q = torch.randn((5, 3, 2, 6, 48), generator=g, device="cuda").bfloat16()[:, :, 1]
    out = torch.full((5, 3, 6, 64), 3.0, device="cuda").bfloat16()
    l5 = _ints([50, 3, 0, 64, 20])
    l5 = torch.minimum(l5, lens)
    got = ll.cache_attention(q, many, l5, out=out[..., :48])
    _check(got, q, many, l5)
    assert bool((out[..., 48:] == 3).all())
    spaced = _empty(1, 64, 2, 48, True, pad=2)
    spaced.copy_(c)
    assert torch.equal(ll.cache_attention(q[:1], spaced, lens)[0], ll.cache_attention(q[:1], c, lens)[0])


# ------------------------------------------------------------------------------- eviction
def _evict_case(N, S, H, d, lens, seed, weights="spread", heads_first=False, pad=0):
    g = _gen(seed)
    c = _empty(N, S, H, d, heads_first, pad)
    c.copy_(torch.randint(0, 256, (N, S, H, d + 16), generator=g, device="cuda").byte())
    if weights == "spread":
        w = torch.exp(3 * torch.randn((N, H, S), generator=g, device="cuda"))
    elif weights == "ties":
        w = torch.randint(0, 4, (N, H, S), generator=g, device="cuda").float() - 1.0
        w[w == 0] = torch.where(torch.rand(int((w == 0).sum()), generator=g, device="cuda") < 0.5, 0.0, -0.0)
    elif weights == "equal":
        w = torch.full((N, H, S), 0.25, device="cuda")
    else:
        w = torch.randn((N, H, S), generator=g, device="cuda")
        w[torch.rand((N, H, S), generator=g, device="cuda") < 0.5] = math.nan
        w[torch.rand((N, H, S), generator=g, device="cuda") < 0.1] = -math.inf
        w[torch.rand((N, H, S), generator=g, device="cuda") < 0.05] = math.inf
    return c, w, _ints(lens)


def _same(a, b):
    return torch.equal(a.view(torch.int32), b.view(torch.int32))


EVICT = [
    # N, S, H, d, lengths, budget, recent, first
    (1, 2, 1, 16, [2], 1, 0, 0), (2, 50, 2, 32, [50, 20], 20, 5, 2), (3, 50, 2, 64, [50, 30, -1], 20, 20, 0),
    (3, 300, 3, 80, [300, 299, 0], 299, 100, 4), (2, 1500, 2, 128, [1500, 1025], 1024, 0, 0),
    (2, 5000, 1, 96, [5000, 7000], 4999, 1, 1), (1, 9000, 2, 128, [9000], 100, 50, 50),
    (4, 40, 1, 112, [40, 39, 38, 37], 37, 3, 30), (1, 70000, 1, 16, [70000], 300, 64, 4),
    (2, 2304, 8, 128, [2304, 2049], 2048, 256, 4), (5, 130, 2, 48, [130, 64, 65, 66, 1], 64, 0, 64),
]


@pytest.mark.parametrize("weights", ["spread", "ties", "equal", "nan"])
@pytest.mark.parametrize("case", EVICT)
def test_evict(case, weights):
    ll = _ll()
    N, S, H, d, lens, budget, recent, first = case
    heads_first = (N + S) % 2 == 0
    c, w, lens = _evict_case(N, S, H, d, lens, S, weights, heads_first, pad=N % 2)
    want, new = plain.evict(w.cpu(), lens.tolist(), budget, recent, first)
    # into another cache
    to, to_w = _empty(N, budget + 3, H, d, not heads_first), torch.full((N, H, budget + 3), 5.0, device="cuda")
    c0, w0 = c.clone(), w.clone()
    kept, new_len = ll.cache_evict(c, w, lens, budget, recent=recent, first=first, into=to, into_weights=to_w)
    assert torch.equal(kept.cpu(), want) and torch.equal(new_len.cpu(), new)
    assert torch.equal(c, c0) and _same(w, w0)
    there = (want >= 0).cuda()
    at = kept.clamp(min=0).long()
    n, h = torch.arange(N, device="cuda")[:, None, None], torch.arange(H, device="cuda")[:, None]
    records = torch.where(there[..., None], c0[n, at, h], 0x7F)
    assert torch.equal(to[:, :budget].transpose(1, 2), records) and bool((to[:, budget:] == 0x7F).all())
    moved = torch.where(there, torch.gather(w0, 2, at), 5.0)
    assert _same(to_w[..., :budget].contiguous(), moved) and bool((to_w[..., budget:] == 5).all())
    # in place: what lies behind the new length is not told, but nothing else is touched
    kept, new_len = ll.cache_evict(c, w, lens, budget, recent=recent, first=first)
    assert torch.equal(kept.cpu(), want) and torch.equal(new_len.cpu(), new)
    room = c[:, :budget].transpose(1, 2)
    assert torch.equal(room[there], records[there])
    assert _same(w[..., :budget][there], moved[there])
    assert torch.equal(c[:, budget:], c0[:, budget:]) and _same(w[..., budget:], w0[..., budget:])
    assert torch.equal(room[~there], c0[:, :budget].transpose(1, 2)[~there])
    if c._base is not None and N % 2:
        assert bool((c._base[..., d + 16:] == 0x7F).all())


def test_evict_twice_does_nothing_more():
    ll = _ll()
    c, w, lens = _evict_case(2, 400, 2, 64, [400, 150], 1)
    _, new = ll.cache_evict(c, w, lens, 200, recent=50, first=4)
    c0, w0 = c.clone(), w.clone()
    kept, again = ll.cache_evict(c, w, new, 200, recent=50, first=4)
    assert torch.equal(c, c0) and torch.equal(w, w0) and torch.equal(again, new)
    assert kept[0, 0].tolist() == list(range(200)) and kept[1, 1].tolist() == list(range(150)) + [-1] * 50


# ------------------------------------------------------------------------------- together
def test_a_decoding_run():
    """Prompt, drafted blocks of which a part is taken, evictions between: the cache's calls as a program
    makes them, against the same steps in 64 bits on lists of positions."""
    ll = _ll()
    N, H, Hq, d, S, budget, T = 3, 2, 8, 64, 160, 96, 4
    g = _gen(77)
    cache = _empty(N, S, H, d, True)
    w = torch.full((N, H, S), math.nan, device="cuda")
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    prompt = _ints([100, 60, 130])
    k, v = rnd(N, 130, H, d), rnd(N, 130, H, d)
    ll.cache_append(cache, k, v, prompt, weights=w)
    sim = [[dict(k=plain.round_values(k[n, 130 - L:, h]), v=plain.round_values(v[n, 130 - L:, h]),
                 w=torch.zeros(L, dtype=torch.float64, device="cuda")) for h in range(H)]
           for n, L in enumerate(prompt.tolist())]
    lens = prompt.clone()
    ws = None
    for step in range(12):
        k, v, q = rnd(N, T, H, d), rnd(N, T, H, d), rnd(N, T, Hq, d)
        lens = lens + T
        ll.cache_append(cache, k, v, lens, weights=w)
        ws = ws or ll.Workspace(ll.cache_attention_workspace_bytes(q, cache))
        out, lse = ll.cache_attention(q, cache, lens, weights=w, ws=ws)
        taken = torch.randint(1, T + 1, (N,), generator=g, device="cuda").int()
        for n in range(N):
            for h in range(H):
                s = sim[n][h]
                s["k"] = torch.cat([s["k"], plain.round_values(k[n, :, h])])
                s["v"] = torch.cat([s["v"], plain.round_values(v[n, :, h])])
                s["w"] = torch.cat([s["w"], torch.zeros(T, dtype=torch.float64, device="cuda")])
                for t in range(T):
                    m = len(s["w"]) - (T - 1 - t)
                    x = q[n, t, h * 4:h * 4 + 4].double() @ s["k"][:m].T * d ** -0.5
                    p = torch.softmax(x, 1)
                    o, A = p @ s["v"][:m], p @ s["v"][:m].abs()
                    off = (out[n, t, h * 4:h * 4 + 4].double() - o).abs()
                    assert bool((off <= 2.0 ** -9 * A + 2.0 ** -8 * o.abs()).all())
                    off = (lse[n, t, h * 4:h * 4 + 4].double() - torch.logsumexp(x, 1)).abs()
                    assert bool((off <= 2.0 ** -15).all())
                    s["w"][:m] += p.sum(0)
        lens = lens - T + taken                      # the others are written over by the next block
        for n in range(N):
            for h in range(H):
                s = sim[n][h]
                for name in s:
                    s[name] = s[name][:int(lens[n])]
        if step % 3 == 2:
            kept, lens = ll.cache_evict(cache, w, lens, budget, recent=16, first=2)
            for n in range(N):
                for h in range(H):
                    s, at = sim[n][h], kept[n, h][kept[n, h] >= 0].long()
                    L = len(s["w"])
                    assert len(at) == min(L, budget)
                    # what stays is what has the largest weights, up to their rounding
                    rest = torch.ones(L, dtype=torch.bool, device="cuda")
                    rest[at] = False
                    rest[:2] = rest[max(L - 16, 0):] = False
                    inner = at[(at >= 2) & (at < L - 16)]
                    if bool(rest.any()) and len(inner):
                        assert float(s["w"][inner].min()) >= float(s["w"][rest].max()) * (1 - 2.0 ** -12)
                    for name in s:
                        s[name] = s[name][at]
    for n in range(N):
        for h in range(H):
            L = int(lens[n])
            got = w[n, h, :L].double()
            assert bool(((got - sim[n][h]["w"]).abs() <= 2.0 ** -12 * (1 + sim[n][h]["w"])).all())
    assert ws.status() == 0


def test_beams_reorder_a_cache():
    """The records of beams move like any other state."""
    ll = _ll()
    g = _gen(2)
    cache = torch.randint(0, 256, (2, 3, 20, 2, 80), generator=g, device="cuda").byte()
    parents = _ints([[2, 0, 0], [1, 1, 2]])
    want = torch.stack([cache[r, parents[r].long()] for r in range(2)])
    ll.beam_reorder(cache, parents)
    assert torch.equal(cache, want)


@pytest.mark.parametrize("T,Hq,S", [(2, 8, 600), (2, 8, 3000), (16, 16, 1500)])
def test_captured_and_replayed(T, Hq, S):
    """The four calls in one graph, on another stream, replayed for other contents and lengths."""
    ll = _ll()
    N, H, d, budget = 2, 2, 128, 400
    g = _gen(12)
    lens = _ints([S, 380])
    cache = _filled(ll, g, N, S, H, d, lens)
    k = torch.randn((N, T, H, d), generator=g, device="cuda").bfloat16()
    v, q = torch.randn_like(k), torch.randn((N, T, Hq, d), generator=g, device="cuda").bfloat16()
    w = torch.rand((N, H, S), generator=g, device="cuda")
    ws = ll.Workspace(ll.cache_attention_workspace_bytes(q, cache))

    def step():
        ll.cache_append(cache, k, v, lens, weights=w)
        out, lse = ll.cache_attention(q, cache, lens, weights=w, ws=ws)
        back = ll.cache_read(cache, lens, T)
        return (out, lse, *back, *ll.cache_evict(cache, w, lens, budget, recent=40, first=1))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    start = (cache.clone(), w.clone())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            outs = step()
    for new in ([S, 380], [0, 1], [-1, 599], [401, 2]):
        lens.copy_(_ints(new))
        cache.copy_(start[0])
        w.copy_(start[1])
        k.copy_(torch.randn(k.shape, generator=g, device="cuda"))
        outs[0].fill_(9)
        outs[1].fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        got, state = [o.clone() for o in outs], (cache.clone(), w.clone())
        cache.copy_(start[0])
        w.copy_(start[1])
        want = step()
        torch.cuda.synchronize()
        for a, b, at in zip(got, want, range(6)):
            if at < 2 and new[0] < 0:
                a, b = a[1:], b[1:]
            if a.is_floating_point():                # positions that nobody wrote are NaN, on both sides
                a, b = a.nan_to_num(7e7), b.nan_to_num(7e7)
            assert torch.equal(a, b), (new, at)
        assert torch.equal(state[0], cache) and torch.equal(state[1], w)


def test_calls_at_once_on_two_streams():
    """Each with a workspace of its own: the few rows' kernel, the many rows', weights and evictions side by side."""
    ll = _ll()
    jobs = []
    for i, (N, T, Hq, H, d, S) in enumerate([(3, 16, 32, 8, 128, 2500), (2, 1, 32, 8, 128, 9000)]):
        q, c, lens, w = _case(ll, N, T, Hq, H, d, S, "bf16", 40 + i)
        ws = ll.Workspace(ll.cache_attention_workspace_bytes(q, c))

        def job(q=q, c=c, lens=lens, w=w, ws=ws):
            w1, c1 = w.clone(), c.clone()
            got = ll.cache_attention(q, c1, lens, weights=w1, ws=ws)
            return (*got, w1.clone(), *ll.cache_evict(c1, w1, lens, 700, recent=30, first=2), *ll.cache_read(c1, lens, 5))

        jobs.append((job, job(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    results = []
    for _ in range(10):
        for job, want, stream in jobs:
            with torch.cuda.stream(stream):
                results.append((want, job()))
    torch.cuda.synchronize()
    for want, got in results:
        for a, b in zip(want, got):
            assert torch.equal(a.nan_to_num(7e7), b.nan_to_num(7e7)) if a.is_floating_point() else torch.equal(a, b)


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes: the last sequence's records lie behind them."""
    ll = _ll()
    N, S, H, d = 5, 1 << 20, 6, 128                  # 4.5 GB
    cache = torch.empty((N, S, H, d + 16), dtype=torch.uint8, device="cuda")
    cache[:, :64] = 0x7F
    g = _gen(8)
    lens = _ints([1, 0, -1, 2, S])
    k = torch.randn((N, 3, H, d), generator=g, device="cuda").bfloat16()
    cache[4, S - 64:] = 0
    cache[4, :S - 3] = 0
    ll.cache_append(cache, k, k, lens)
    got = ll.cache_read(cache, lens, 3)
    want = plain.round_values(k)
    want[0, :2], want[1], want[2], want[3, :1] = 0, 0, 0, 0
    assert torch.equal(got[0].double(), want) and torch.equal(got[1].double(), want)
    # all keys but the last three are 0: their scores are 0 and their values too
    q = torch.randn((N, 1, H, d), generator=g, device="cuda").bfloat16()
    out, lse = ll.cache_attention(q, cache, lens)
    s = torch.einsum("hd,jhd->hj", q[4, 0].double(), want[4]) * d ** -0.5
    total = torch.exp(s).sum(1) + (S - 3)
    assert bool(((lse[4, 0].double() - torch.log(total)).abs() <= 2.0 ** -16 + 2.0 ** -19).all())
    o = torch.einsum("hj,jhd->hd", torch.exp(s) / total[:, None], want[4])
    A = torch.einsum("hj,jhd->hd", torch.exp(s) / total[:, None], want[4].abs())
    assert bool(((out[4, 0].double() - o).abs() <= 2.0 ** -9 * A + 2.0 ** -8 * o.abs()).all())


def test_tensors_elsewhere_are_refused():
    ll = _ll()
    c, w, lens = _empty(1, 4, 1, 32), torch.zeros(1, 1, 4, device="cuda"), _ints([4])
    k = torch.zeros(1, 1, 1, 32, device="cuda")
    for bad in (dict(cache=c.cpu()), dict(cache=c.int()), dict(cache=c[..., :31]), dict(cache=c[0]),
                dict(cache=c[..., ::2]), dict(k=k.cpu()), dict(k=k[0]), dict(k=k[..., :16]), dict(v=k.bfloat16()),
                dict(seq_len=lens.cpu()), dict(seq_len=lens.long()), dict(seq_len=_ints([1, 2])),
                dict(weights=w.double()), dict(weights=w[..., :3]), dict(weights=w.cpu()), dict(k_unit=3.0),
                dict(k=k.half(), v=k.half())):
        args = {**dict(cache=c, k=k, v=k, seq_len=lens, weights=w), **bad}
        with pytest.raises((ValueError, ll.LilicorrError)):
            ll.cache_append(**args)
    for bad in (dict(q=k.cpu()), dict(q=k[..., :16]), dict(q=k.half()), dict(out=torch.zeros_like(k).bfloat16()),
                dict(lse=torch.zeros(1, 1, 2, device="cuda")), dict(weights=w[:, :, :2]), dict(scale=0.0),
                dict(ws=ll.Workspace(256, device="cpu"))):
        args = {**dict(q=k, cache=c, seq_len=lens), **bad}
        with pytest.raises((ValueError, ll.LilicorrError)):
            ll.cache_attention(**args)
    for bad in (dict(budget=0), dict(budget=2, recent=3), dict(into=_empty(1, 4, 1, 32)),
                dict(into_weights=w.clone()), dict(into=c, into_weights=w),
                dict(into=_empty(1, 1, 1, 32), into_weights=w[..., :1].contiguous()),
                dict(into=_empty(1, 4, 1, 48), into_weights=w.clone()), dict(weights=w[:, :, ::2])):
        args = {**dict(cache=c, weights=w, seq_len=lens, budget=2), **bad}
        with pytest.raises((ValueError, ll.LilicorrError)):
            ll.cache_evict(**args)
    with pytest.raises((ValueError, ll.LilicorrError)):
        ll.cache_read(c, lens, -1)
    with pytest.raises((ValueError, ll.LilicorrError)):
        ll.cache_read(c, lens, 1, dtype=torch.float16)
