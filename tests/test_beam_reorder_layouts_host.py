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
