"""CPU checks of the beam calls: shape and argument errors come back before anything is enqueued."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_20530_gb300 as ll
    return ll.lib()


def _select(lib, dtype=0, R=1, W=2, V=100, n=4, end_id=-1, done=None, ptr=None, ws=None, ws_bytes=0):
    return lib.lilicorr_beam_select(ptr, dtype, R, W, V, n, ptr, done, end_id, ptr, ptr, ptr, None,
                                    ws, ws_bytes, None)


def test_beam_select_refusals(lib):
    assert _select(lib, dtype=5) == 3
    for bad in (dict(W=0), dict(W=65), dict(n=0), dict(n=33), dict(V=0), dict(V=1, n=3), dict(R=-1),
                dict(R=40000, W=2)):
        assert _select(lib, **bad) == 2, bad
    p = ctypes.c_void_p(4096)                       # never read: the calls are refused before
    assert _select(lib, end_id=-2, ptr=p, ws=p, ws_bytes=1 << 30) == 1
    assert _select(lib, end_id=100, ptr=p, ws=p, ws_bytes=1 << 30) == 1
    assert _select(lib, done=p, ptr=p, ws=p, ws_bytes=1 << 30) == 1      # done without an end token
    assert _select(lib, R=0) == 0
    assert _select(lib) == 1                        # null pointers
    assert _select(lib, ptr=ctypes.c_void_p(4100), ws=p, ws_bytes=1 << 30) == 1   # misaligned
    assert _select(lib, ptr=p, ws=p, ws_bytes=256) == 7
    need = lib.lilicorr_beam_select_workspace_bytes
    assert need(1, 2, 100, 4) > 256 and need(1, 2, 100, 33) == 0 and need(1, 65, 100, 4) == 0
    assert need(1, 1, 3, 4) == 0 and need(1, 2, 3, 4) > 0


def test_beam_merge_refusals(lib):
    def f(R=1, W=2, K=4, n=4, end_id=-1, done=None, p=None):
        return lib.lilicorr_beam_merge(p, p, R, W, K, n, p, done, end_id, p, p, p, None, None, None)
    for bad in (dict(W=0), dict(W=65), dict(K=0), dict(K=33), dict(n=9), dict(n=33, K=32), dict(n=0),
                dict(R=-1)):
        assert f(**bad) == 2, bad
    p = ctypes.c_void_p(4096)
    assert f(end_id=-2, p=p) == 1 and f(done=p, p=p) == 1
    assert f(R=0) == 0
    assert f() == 1


def test_beam_reorder_refusals(lib):
    p = (ctypes.c_void_p * 1)(4096)
    par = ctypes.c_void_p(4096)

    def f(states=p, n=1, R=1, W=2, S=3, H=1, row=16, parents=par):
        return lib.lilicorr_beam_reorder(states, n, R, W, S, H, row, 96, 48, 16, 16, parents, None,
                                         None)
    for bad in (dict(n=-1), dict(R=-1), dict(R=65536), dict(W=0), dict(W=65), dict(S=-1), dict(H=-1),
                dict(row=1 << 32), dict(S=1 << 30, row=64), dict(S=1 << 30, row=6)):
        assert f(**bad) == 2, bad
    for none in (dict(n=0), dict(R=0), dict(S=0), dict(H=0), dict(row=0)):
        assert f(**none) == 0, none
    assert f(states=None) == 1 and f(parents=None) == 1
    assert f(states=(ctypes.c_void_p * 1)(None)) == 1


def test_beam_reorder_refuses_arrays_that_overlap(lib):
    """No byte may belong to two rows: the stride nest and its pairs against the sets of bytes."""
    import itertools
    import random
    rng = random.Random(7)

    def cells(at, extents, strides, row):
        return [at + sum(i * s for i, s in zip(idx, strides)) + b
                for idx in itertools.product(*map(range, extents)) for b in range(row)]

    def refused(at, extents, strides, row):
        return lib.lilicorr_test_states_overlap((ctypes.c_void_p * len(at))(*at), len(at),
                                                (ctypes.c_int64 * 4)(*strides),
                                                (ctypes.c_int64 * 4)(*extents), ctypes.c_size_t(row))

    seen = [0, 0]
    for _ in range(400):
        row = rng.choice((1, 2, 4))
        extents = [rng.randint(1, 4) for _ in range(4)]
        order = list(range(4))
        rng.shuffle(order)
        strides, span = [0] * 4, row
        for d in order:                                        # a slice of a dense array, or nearly
            strides[d] = (span + rng.choice((0, 0, 1, 3))) * rng.choice((1, 1, 1, -1))
            span += (extents[d] - 1) * abs(strides[d])
        one = cells(0, extents, strides, row)
        assert len(set(one)) == len(one)
        delta = rng.randint(-span - 2, span + 2)
        both = one + cells(delta, extents, strides, row)
        want = int(len(set(both)) < len(both))
        assert refused([5000, 5000 + delta], extents, strides, row) == want, (extents, strides, delta)
        assert refused([5000], extents, strides, row) == 0
        seen[want] += 1
    assert min(seen) > 50
    assert refused([4096], (2, 2, 1, 1), (0, 64, 0, 0), 64) == 1    # one array for all requests
    assert refused([4096], (1, 2, 3, 1), (0, 0, 64, 0), 64) == 1    # beams that share their rows
    assert refused([4096], (1, 1, 3, 1), (0, 0, 48, 0), 64) == 1
    assert refused([4096, 8192, 4096], (1, 2, 3, 1), (0, 192, 64, 0), 64) == 1


def test_beam_reorder_call_refuses_them(lib):
    p = ctypes.c_void_p(4096)

    def f(at, strides):
        return lib.lilicorr_beam_reorder((ctypes.c_void_p * len(at))(*at), len(at), 2, 2, 3, 1, 16,
                                         *strides, p, None, None)
    assert f([4096, 4096], (96, 48, 16, 0)) == 1
    assert f([4096], (0, 48, 16, 0)) == 1
    assert f([4096], (96, 0, 16, 0)) == 1
    assert f([4096], (96, 32, 16, 0)) == 1
