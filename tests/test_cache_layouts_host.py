"""CPU checks of layouts that calls on a 4-bit cache accept: nothing is enqueued by the calls made here."""
import ctypes

import pytest

import test_cache_host as base
from test_cache_host import ll  # noqa: F401


@pytest.mark.parametrize("stride", [(16000, 160, 64), (16000, 0, 80), (160, 160, 64)])
def test_evict_from_records_that_overlap(ll, stride):  # noqa: F811
    """A cache that is read may share its records between heads, positions and sequences; one that is written may
    not. (Of no sequences, so that there is nothing to do.)"""
    shared = base._cache(ll, sequences=0, stride=stride)
    there = dict(into_cache=base.Q, into_weights=ctypes.c_void_p(1 << 41))
    assert base._evict(ll, shared, into=base._cache(ll, sequences=0), **there) == 0
    assert base._evict(ll, shared) == 1
    assert base._evict(ll, base._cache(ll, sequences=0), into=shared, **there) == 1
