"""CPU checks of prefix_attention: shapes, strides and arguments are refused before anything is
enqueued, and the workspace grows with the call."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def ll():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_20530_gb300 as ll
    return ll


def _desc(ll, **kw):
    base = dict(groups=2, beams=3, tokens=1, q_heads=8, kv_heads=2, head_dim=64, prefix_capacity=100,
                own_capacity=20, dtype=ll.BF16, scale=0.125)
    base.update({k: v for k, v in kw.items() if not k.endswith("_stride")})
    x = ll.PrefixAttentionDesc(**base)
    d, Hq, Hkv = base["head_dim"], base["q_heads"], base["kv_heads"]
    for name, strides in (("q_stride", (Hq * d, Hq * d, d)), ("out_stride", (Hq * d, Hq * d, d)),
                          ("prefix_k_stride", (100 * Hkv * d, Hkv * d, d)),
                          ("prefix_v_stride", (100 * Hkv * d, Hkv * d, d)),
                          ("k_stride", (20 * Hkv * d, Hkv * d, d)),
                          ("v_stride", (20 * Hkv * d, Hkv * d, d))):
        getattr(x, name)[:] = kw.get(name, strides)
    return x


P = ctypes.c_void_p(4096)                       # never read: the calls are refused before
NAMES = ("q", "prefix_k", "prefix_v", "prefix_len", "k", "v", "seq_len", "out", "lse", "ws")


def _call(ll, x, ws_bytes=1 << 40, **ptrs):
    return ll.lib().lilicorr_prefix_attention(ctypes.byref(x), *(ptrs.get(n, P) for n in NAMES),
                                              ws_bytes, None)


def test_shapes_are_refused(ll):
    assert _call(ll, _desc(ll, dtype=7)) == 3
    for bad in (dict(groups=-1), dict(beams=0), dict(tokens=0), dict(q_heads=0), dict(kv_heads=0),
                dict(q_heads=9), dict(head_dim=0), dict(head_dim=4), dict(head_dim=60),
                dict(head_dim=136), dict(prefix_capacity=-1), dict(own_capacity=-1),
                dict(prefix_capacity=(1 << 30) + 1), dict(beams=1 << 30)):
        x = _desc(ll, **bad)
        assert _call(ll, x) == 2, bad
        assert ll.lib().lilicorr_prefix_attention_workspace_bytes(ctypes.byref(x)) == 0, bad


def test_arguments_are_refused(ll):
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert _call(ll, _desc(ll, scale=scale)) == 1
    for name in NAMES:
        assert _call(ll, _desc(ll), **{name: None}) == 1, name
    odd = ctypes.c_void_p(4104)
    for name in ("q", "prefix_k", "prefix_v", "k", "v", "out", "ws"):
        assert _call(ll, _desc(ll), **{name: odd}) == 1, name
    for name in ("q_stride", "out_stride", "prefix_k_stride", "prefix_v_stride", "k_stride", "v_stride"):
        good = list(getattr(_desc(ll), name))
        for i, v in ((0, good[0] + 4), (2, -64), (2, 1 << 41)):
            s = list(good)
            s[i] = v
            assert _call(ll, _desc(ll, **{name: s})) == 1, (name, s)
    assert ll.lib().lilicorr_prefix_attention(None, *([P] * 10), 1 << 40, None) == 1
    assert _call(ll, _desc(ll, groups=0)) == 0                   # nothing to do
    x = _desc(ll)
    need = ll.lib().lilicorr_prefix_attention_workspace_bytes(ctypes.byref(x))
    assert need > 256 and _call(ll, x, ws_bytes=need - 1) == 7


def test_out_that_overlaps_itself_is_refused(ll):
    """Every row of ``out`` is written by somebody; caches may be shared, and are read."""
    for s in ((0, 512, 64), (512, 512, 0), (512, 512, 56), (448, 512, 64)):
        assert _call(ll, _desc(ll, out_stride=s), ws_bytes=16) == 1, s
    for s in ((512, 512, 64), (64, 512, 6 * 64), (1024, 8, 64), (520, 0, 64)):
        assert _call(ll, _desc(ll, out_stride=s), ws_bytes=16) == 7, s
    assert _call(ll, _desc(ll, prefix_k_stride=(0, 128, 64), prefix_v_stride=(0, 128, 64)),
                 ws_bytes=16) == 7


def test_strides_of_single_entries_do_not_count(ll):
    """A dimension of one has no stride: the refusal that comes next is the workspace's."""
    x = _desc(ll, q_stride=(512, 3, 64), out_stride=(512, -5, 64))
    assert _call(ll, x, ws_bytes=16) == 7


def test_workspace_grows_with_the_call(ll):
    f = lambda **kw: ll.lib().lilicorr_prefix_attention_workspace_bytes(  # noqa: E731
        ctypes.byref(_desc(ll, **kw)))
    assert f(beams=1) < f(beams=300) and f(tokens=1) < f(tokens=40)
    assert f(prefix_capacity=0, own_capacity=0) < f()
