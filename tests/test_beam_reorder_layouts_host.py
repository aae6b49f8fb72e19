"""CPU checks of lilicorr_beam_reorder_layouts: all layouts are looked at, in whatever order they come,
before anything is enqueued."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def ll():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_20530_gb300 as ll
    return ll


def _layout(ll, at, positions=3, heads=1, row=16, strides=(96, 48, 16, 0), n=None):
    return ll.BeamStates((ctypes.c_void_p * max(1, len(at)))(*at), len(at) if n is None else n, positions, heads,
                         row, *strides)


def _call(ll, layouts, R=1, W=2, n=None, parents=4096):
    arr = (ll.BeamStates * max(1, len(layouts)))(*layouts)
    return ll.lib().lilicorr_beam_reorder_layouts(arr if layouts else None, len(layouts) if n is None else n, R, W,
                                                  ctypes.c_void_p(parents) if parents else None, None, None)


def test_a_refused_layout_refuses_the_call(ll):
    good = _layout(ll, [4096])                      # would launch (and fail here, without a GPU: status 4)
    for bad, status in ((_layout(ll, [8192], positions=-1), 2), (_layout(ll, [8192], heads=-1), 2),
                        (_layout(ll, [8192], n=-1), 2), (_layout(ll, [8192], row=1 << 32), 2),
                        (_layout(ll, [8192], positions=1 << 30, row=64), 2), (_layout(ll, [None]), 1),
                        (_layout(ll, [8192, 8192]), 1), (_layout(ll, [8192], strides=(96, 32, 16, 0)), 1)):
        assert _call(ll, [bad]) == status
        assert _call(ll, [good, bad]) == status
        assert _call(ll, [bad, good]) == status
        assert _call(ll, [good, _layout(ll, [16384], row=8), bad]) == status


def test_sizes_and_pointers(ll):
    good = _layout(ll, [4096])
    assert _call(ll, [good], n=-1) == 2 and _call(ll, [good], R=-1) == 2 and _call(ll, [good], R=65536) == 2
    assert _call(ll, [good], W=0) == 2 and _call(ll, [good], W=65) == 2
    assert _call(ll, [], n=1) == 1 and _call(ll, [good], parents=None) == 1
    assert _call(ll, []) == 0
    # layouts with nothing to move
    none = [_layout(ll, [4096], positions=0), _layout(ll, [4096], heads=0), _layout(ll, [4096], row=0), _layout(ll, [])]
    assert _call(ll, none) == 0 and _call(ll, none, parents=None) == 0
    assert _call(ll, [good] + none, R=0) == 0


def _overlap(ll, layouts, R, W):
    arr = (ll.BeamStates * len(layouts))(*layouts)
    return ll.lib().lilicorr_test_layouts_overlap(arr, len(layouts), R, W)


def test_arrays_of_different_layouts_that_share_bytes(ll):
    """Random pairs of layouts, some cut from one buffer and some with nothing in common, against the
    sets of their bytes."""
    import itertools
    import random
    rng = random.Random(11)

    def cells(at, extents, strides, row):
        return {at + sum(i * s for i, s in zip(idx, strides)) + b
                for idx in itertools.product(*map(range, extents)) for b in range(row)}

    def nest(R, W):
        row, ext = rng.choice((1, 2, 3, 8)), [R, W, rng.randint(1, 4), rng.randint(1, 3)]
        order, strides, span = list(range(4)), [0] * 4, row
        rng.shuffle(order)
        for d in order:
            strides[d] = (span + rng.choice((0, 0, 1, 5))) * rng.choice((1, 1, 1, -1))
            span += (ext[d] - 1) * abs(strides[d])
        return ext, strides, row, span

    seen = [0, 0]
    for turn in range(1500):
        R, W = rng.randint(1, 3), rng.randint(1, 3)
        ext, strides, row, span = nest(R, W)
        if turn % 2:                                           # the same buffer: fewer positions, part of the rows
            ext2, strides2 = list(ext), list(strides)
            ext2[2], row2 = rng.randint(1, ext[2]), rng.randint(1, row)
        else:
            ext2, strides2, row2, _ = nest(R, W)
        delta = rng.randint(-span - 4, span + 4)
        a, b = cells(0, ext, strides, row), cells(delta, ext2, strides2, row2)
        base = 1 << 20
        x = _layout(ll, [base], ext[2], ext[3], row, strides)
        y = _layout(ll, [base + delta], ext2[2], ext2[3], row2, strides2)
        want = int(bool(a & b))
        assert _overlap(ll, [x, y], R, W) == want and _overlap(ll, [y, x], R, W) == want, (ext, strides, delta)
        seen[want] += 1
    assert min(seen) > 300


def test_layouts_cut_from_one_cache(ll):
    """Positions [0, 64) and [32, 100) of one cache share 32 of them; [0, 64) and [64, 100) none, and
    neither do keys of 128 and values of 64 bytes that lie beside one another in each head."""
    s = (8 * 100 * 192 * 4, 100 * 192 * 4, 192 * 4, 192)

    def part(p0, p1, off=0, row=192):
        return _layout(ll, [4096 + p0 * s[2] + off], p1 - p0, 4, row, s)
    assert _overlap(ll, [part(0, 64), part(32, 100)], 2, 8) == 1
    assert _call(ll, [part(0, 64), part(32, 100)], R=2, W=8) == 1
    assert _overlap(ll, [part(0, 64), part(64, 100)], 2, 8) == 0
    assert _overlap(ll, [part(0, 100, 0, 128), part(0, 100, 128, 64)], 2, 8) == 0
    assert _overlap(ll, [part(0, 100, 0, 129), part(0, 100, 128, 64)], 2, 8) == 1
    assert _overlap(ll, [part(0, 64, 0, 128), part(32, 100, 128, 64), part(70, 80, 0, 100)], 2, 8) == 0
    assert _overlap(ll, [part(0, 64, 0, 128), part(32, 100, 128, 64), part(70, 80, 100, 29)], 2, 8) == 1


def test_layouts_with_nothing_in_common_end(ll):
    """Two large arrays that interleave without a common stride: told apart, or refused, in a bounded time."""
    import time
    x = _layout(ll, [1 << 30], 1 << 20, 1, 2, (1 << 44, 1 << 40, 1024, 0))
    y = _layout(ll, [(1 << 30) + 512], 1 << 20, 1, 2, (1 << 44, 1 << 40, 1000, 0))
    t = time.perf_counter()
    assert _overlap(ll, [x, y], 8, 64) in (0, 1)
    assert time.perf_counter() - t < 5.0
