"""CPU checks of the calls on a 4-bit cache: shapes, strides and arguments are refused before anything is
enqueued, by the C entries and by the binding."""
import ctypes
import random

import pytest
import torch

from _cache_plain import CODES, SCALES, round_values, values

P = ctypes.c_void_p(4096)                       # never read: the calls are refused before
Q = ctypes.c_void_p(1 << 40)
ODD = ctypes.c_void_p(4104)
I64x3 = ctypes.c_int64 * 3


@pytest.fixture(scope="module")
def ll():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_20530_gb300 as ll
    return ll


def _cache(ll, **kw):
    base = dict(sequences=2, capacity=100, kv_heads=2, head_dim=64, k_unit=1.0, v_unit=1.0)
    base.update({k: v for k, v in kw.items() if k in base})
    x = ll.CacheDesc(**base)
    x.stride[:] = kw.get("stride", (100 * 160, 160, 80))
    return x


BAD_SHAPES = [dict(sequences=-1), dict(capacity=-1), dict(capacity=(1 << 30) + 1), dict(kv_heads=0),
              dict(head_dim=0), dict(head_dim=8), dict(head_dim=72), dict(head_dim=144),
              dict(sequences=1 << 20, kv_heads=1 << 12)]
BAD_ARGS = [dict(k_unit=0.0), dict(k_unit=3.0), dict(v_unit=-1.0), dict(v_unit=float("nan")),
            dict(k_unit=2.0 ** 61), dict(v_unit=2.0 ** -61), dict(k_unit=float("inf")),
            dict(stride=(16000, 160, 72)), dict(stride=(-16000, 160, 80)), dict(stride=(1 << 41, 160, 80)),
            dict(stride=(16000, 168, 80))]
OVERLAPPING = [dict(stride=(0, 160, 80)), dict(stride=(16000, 0, 80)), dict(stride=(16000, 160, 64)),
               dict(stride=(160, 160, 80)), dict(stride=(15920, 160, 80))]
FINE = [dict(), dict(stride=(16000, 80, 8000)), dict(stride=(160, 320, 80)), dict(stride=(32000, 176, 96))]


def test_record_bytes(ll):
    f = ll.cache_record_bytes
    assert [f(d) for d in (16, 64, 80, 96, 128)] == [32, 80, 96, 112, 144]
    assert all(f(d) == 0 for d in (-16, 0, 8, 24, 72, 136, 144, 256))


def _tokens(ll, append, x, T=3, dtype=1, cache=P, k=Q, v=Q, ks=(384, 128, 64), vs=(384, 128, 64), lens=P):
    f = ll.lib().lilicorr_cache_append if append else ll.lib().lilicorr_cache_read
    args = [ctypes.byref(x) if x else None, cache, dtype, T, k, None if ks is None else I64x3(*ks), v,
            None if vs is None else I64x3(*vs), lens] + ([None] if append else []) + [None]
    return f(*args)


@pytest.mark.parametrize("append", [True, False])
def test_append_and_read_refuse(ll, append):
    for bad in BAD_SHAPES:
        assert _tokens(ll, append, _cache(ll, **bad)) == 2, bad
    for bad in BAD_ARGS:
        assert _tokens(ll, append, _cache(ll, **bad)) == 1, bad
    if append:                                       # every record is written by somebody
        for bad in OVERLAPPING:
            assert _tokens(ll, append, _cache(ll, **bad)) == 1, bad
    x = _cache(ll)
    assert _tokens(ll, append, None) == 1
    assert _tokens(ll, append, x, dtype=2) == 3
    assert _tokens(ll, append, x, T=-1) == 2
    assert _tokens(ll, append, x, T=1 << 30) == 2
    for bad in (dict(cache=None), dict(cache=ODD), dict(k=None), dict(v=None), dict(k=ODD), dict(v=ODD),
                dict(ks=None), dict(vs=None), dict(lens=None), dict(ks=(384, 128, 60)),
                dict(vs=(-384, 128, 64)), dict(ks=(384, 128, 1 << 41)), dict(dtype=0, vs=(384, 130, 64))):
        assert _tokens(ll, append, x, **bad) == 1, bad
    if not append:
        for bad in (dict(ks=(0, 128, 64)), dict(vs=(384, 128, 0)), dict(ks=(384, 64, 64))):
            assert _tokens(ll, append, x, **bad) == 1, bad
    assert _tokens(ll, append, x, T=0) == 0          # nothing to do
    assert _tokens(ll, append, _cache(ll, sequences=0)) == 0


def _attend(ll, x, ws_bytes=1 << 40, **kw):
    d = ll.CacheAttentionDesc(cache=x, tokens=kw.get("T", 2), q_heads=kw.get("Hq", 8),
                              dtype=kw.get("dtype", 1), scale=kw.get("scale", 0.125))
    d.q_stride[:] = kw.get("qs", (1024, 512, 64))
    d.out_stride[:] = kw.get("os", (1024, 512, 64))
    names = ("q", "cache", "lens", "out", "lse", "weights", "ws")
    args = [kw.get(n, None if n == "weights" else P) for n in names]
    return ll.lib().lilicorr_cache_attention(ctypes.byref(d), *args, ws_bytes, None), d


def test_attention_refuses(ll):
    for bad in BAD_SHAPES:
        assert _attend(ll, _cache(ll, **bad))[0] == 2, bad
    for bad in BAD_ARGS:
        assert _attend(ll, _cache(ll, **bad))[0] == 1, bad
    for shared in OVERLAPPING[:3]:                   # a cache that is read may be shared
        assert _attend(ll, _cache(ll, **shared), ws_bytes=16)[0] == 7, shared
    x = _cache(ll)
    for bad in (dict(T=0), dict(Hq=0), dict(Hq=7), dict(T=1 << 28, Hq=8), dict(T=(1 << 26) + 1)):
        code, d = _attend(ll, x, **bad)
        assert code == 2, bad
        assert ll.lib().lilicorr_cache_attention_workspace_bytes(ctypes.byref(d)) == 0
    assert _attend(ll, x, dtype=5)[0] == 3
    for scale in (0.0, -1.0, float("inf"), float("nan"), 2.0 ** 100):
        assert _attend(ll, x, scale=scale)[0] == 1, scale
    assert _attend(ll, _cache(ll, k_unit=2.0 ** 50), scale=2.0 ** 50)[0] == 1
    for name in ("q", "cache", "lens", "out", "lse", "ws"):
        assert _attend(ll, x, **{name: None})[0] == 1, name
    for name in ("q", "cache", "out", "ws"):
        assert _attend(ll, x, **{name: ODD})[0] == 1, name
    for bad in (dict(qs=(1024, 512, 60)), dict(os=(-1024, 512, 64)), dict(os=(1024, 0, 64)),
                dict(os=(1024, 512, 56)), dict(qs=(1 << 41, 512, 64)), dict(dtype=0, qs=(1024, 514, 64))):
        assert _attend(ll, x, **bad)[0] == 1, bad
    assert _attend(ll, _cache(ll, sequences=0))[0] == 0
    assert ll.lib().lilicorr_cache_attention(None, *[P] * 7, 1 << 40, None) == 1
    code, d = _attend(ll, x, ws_bytes=16)
    need = ll.lib().lilicorr_cache_attention_workspace_bytes(ctypes.byref(d))
    assert code == 7 and need >= 256 and _attend(ll, x, ws_bytes=need - 1)[0] == 7


def _evict(ll, x, budget=50, recent=10, first=2, into=None, cache=P, weights=P, lens=P, into_cache=None,
           into_weights=None, kept=P, new=Q):
    return ll.lib().lilicorr_cache_evict(ctypes.byref(x) if x else None, cache, weights, lens, budget, recent,
                                         first, ctypes.byref(into) if into else None, into_cache,
                                         into_weights, kept, new, None)


def test_evict_refuses(ll):
    for bad in BAD_SHAPES:
        assert _evict(ll, _cache(ll, **bad)) == 2, bad
    for bad in BAD_ARGS + OVERLAPPING:
        assert _evict(ll, _cache(ll, **bad)) == 1, bad
    x = _cache(ll)
    assert _evict(ll, None) == 1
    for bad in (dict(budget=0), dict(budget=-1), dict(recent=-1), dict(first=-1), dict(recent=49),
                dict(recent=51, first=0), dict(recent=2 ** 31 - 1, first=2 ** 31 - 1), dict(cache=None),
                dict(cache=ODD), dict(weights=None), dict(lens=None), dict(kept=None), dict(new=None),
                dict(into_cache=Q), dict(into_weights=Q)):
        assert _evict(ll, x, **bad) == 1, bad
    # places past 2^30 would pass 32 bits in a stride over them
    assert _evict(ll, x, budget=(1 << 30) + 1) == 2 and _evict(ll, x, budget=2 ** 31 - 1) == 2
    # lengths that all heads read, and one of them would write
    assert _evict(ll, x, new=ctypes.c_void_p(4100)) == 1 and _evict(ll, x, lens=Q, new=Q) == 1
    there = dict(into_cache=Q, into_weights=ctypes.c_void_p(1 << 41), new=Q)
    for bad in (dict(sequences=3), dict(kv_heads=1), dict(head_dim=80), dict(capacity=49),
                dict(capacity=-1)):
        assert _evict(ll, x, into=_cache(ll, **bad), **there) == 2, bad
    for bad in (dict(k_unit=2.0), dict(v_unit=0.5), dict(stride=(0, 160, 80))):
        assert _evict(ll, x, into=_cache(ll, **bad), **there) == 1, bad
    y = _cache(ll)
    for bad in (dict(into_cache=None), dict(into_cache=ODD), dict(into_weights=None),
                dict(into_cache=ctypes.c_void_p(4096 + 31984)),      # the last 16 bytes of the cache
                dict(into_weights=ctypes.c_void_p(4096 + 4 * 399))):
        assert _evict(ll, x, into=y, **{**there, **bad}) == 1, bad
    assert _evict(ll, _cache(ll, sequences=0)) == 0


def test_binding_refuses(ll):
    """The binding checks what the C entries cannot see; on a CPU tensor it says so."""
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        ll.cache_append(torch.zeros(1, 4, 1, 32, dtype=torch.uint8), torch.zeros(1, 1, 1, 16),
                        torch.zeros(1, 1, 1, 16), torch.zeros(1, dtype=torch.int32))


def test_plain_rounding():
    """The tests' own rounding: values that the records hold stay, and no other is nearer."""
    r = random.Random(5)
    x = torch.tensor([[r.uniform(-8, 8) * 2.0 ** r.randint(-12, 9) for _ in range(64)] for _ in range(50)])
    y = round_values(x)
    assert torch.equal(round_values(y), y)
    g = x.double().unflatten(-1, (-1, 16))
    top = g.abs().amax(-1, keepdim=True)
    s = torch.tensor(SCALES[1:127], dtype=torch.float64)
    best = s[(top / 6 - s).abs().argmin(-1)][..., None]
    grid = torch.tensor(CODES, dtype=torch.float64) * best[..., None]
    off = (g.abs()[..., None] - grid).abs().amin(-1).flatten(-2)
    assert torch.equal((x.double() - y).abs(), off)
    half = torch.zeros(1, 16, dtype=torch.uint8)
    half[0, :8] = torch.tensor([0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE])
    half[0, 8] = 0x38                                # a scale of 1
    assert values(half)[0].tolist() == CODES + [-c for c in CODES]
